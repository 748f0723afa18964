// c = act(a b + bias) + residual on the matrix cores.
//
// A work-group of four wavefronts has a tile of 64 x 64 of c and walks along k in steps of 32.  Each thread brings eight
// neighbouring elements of either operand through registers into LDS, the next step's while the matrix instructions run
// on this one's; both operands lie in LDS with k last, so that an instruction's operand is one 16-byte read of a lane.
// A wavefront has 16 rows of the tile: four v_mfma_f32_16x16x32 a step, with the operands exchanged, so that a lane's
// four results are neighbouring columns of one row.  The sums go through LDS once more, to leave a thread eight
// neighbouring columns for the epilogue: the bias, the checkpoint of z (four lanes hold a group of 32), the activation, the
// residual and the one rounding.

#include <type_traits>

#include "ds_ops.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

// An operand: element (p, k), p a row of a or a column of b.
struct Operand {
  const void *base;
  int64_t ld;      // elements from p to p + 1 (k_last), or from k to k + 1
  int64_t extent;  // of p
  const uint8_t *scale;
  int64_t scale_stride;
  bool k_last;  // neighbouring k are neighbours in memory
};

struct Epilogue {
  Rows c, residual, saved;
  const void *bias;
  int64_t m, n;
  uint32_t c_dtype, bias_dtype, act;
};

__device__ inline f32x4 mfma(u32x4 x, u32x4 y, f32x4 sum, __hip_bfloat16) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), sum, 0, 0, 0);
}
__device__ inline f32x4 mfma(u32x4 x, u32x4 y, f32x4 sum, __half) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), sum, 0, 0, 0);
}

__device__ inline float activation_any(float z, uint32_t act) {
  switch (act) {
    case DS_ACT_GELU: return activation<DS_ACT_GELU>(z);
    case DS_ACT_GELU_TANH: return activation<DS_ACT_GELU_TANH>(z);
    case DS_ACT_SILU: return activation<DS_ACT_SILU>(z);
    default: return z;
  }
}

// Eight sums of row i from column j (a multiple of 8) on, n <= 8 of them in c, leave by the epilogue.  All lanes of the wavefront
// take part, four neighbouring ones with a group of 32 columns.
__device__ inline void finish8(const Epilogue &e, int64_t i, int64_t j, int n, Eight z) {
  if (e.bias) {
    const Eight b = get_up_to8_any(e.bias, e.bias_dtype, j, n, 0.f);
#pragma unroll
    for (int k = 0; k < 8; ++k) z.v[k] += b.v[k];
  }
  if (e.saved.base) {
    Eight s = z;
    if (n < 8) {
#pragma unroll
      for (int k = 0; k < 8; ++k) s.v[k] = k < n ? z.v[k] : 0.f;
    }
    mx8_put(e.saved, i, j, n, s);
  }
  if (e.act != DS_ACT_NONE) {
#pragma unroll
    for (int k = 0; k < 8; ++k) z.v[k] = activation_any(z.v[k], e.act);
  }
  if (n <= 0) return;
  const int64_t at = i * e.c.stride + j, from = i * e.residual.stride + j;
  const auto store = [&](auto type) {
    typedef decltype(type) T;
    if (e.residual.base) {
      const Eight r = get_up_to8<T>(e.residual.base, from, n);
#pragma unroll
      for (int k = 0; k < 8; ++k) z.v[k] += r.v[k];
    }
    put_up_to8<T>(e.c.base, at, n, z);
  };
  if (e.c_dtype == DS_F32) store(float());
  else if (e.c_dtype == DS_BF16) store(__hip_bfloat16());
  else store(__half());
}

constexpr int kTile = 64, kDeep = 32, kPitch = kDeep + 8;

// Eight neighbouring elements of an operand for the LDS: of one p from k on (k_last), or of one k from p on.  Those beyond
// the matrix are 0.
template <typename T>
__device__ inline u32x4 bring8(const Operand &o, int64_t p, int64_t k, int64_t depth) {
  const int64_t line = o.k_last ? p : k, at = o.k_last ? k : p;
  const int64_t lines = o.k_last ? o.extent : depth, length = o.k_last ? depth : o.extent;
  const int64_t left = line < lines ? length - at : 0;
  const int n = (int)(left < 0 ? 0 : left < 8 ? left : 8);
  if (o.scale) {
    const Rows rows{const_cast<void *>(o.base), o.ld, const_cast<uint8_t *>(o.scale), o.scale_stride};
    const Eight e = RowsOf<Mx8>::get(rows, line, at, n);
    u32x4 r;
    Elem<T>::put8(&r, 0, e);
    return r;
  }
  u32x4 r = {0, 0, 0, 0};
  const uint16_t *q = (const uint16_t *)o.base + line * o.ld + at;
  if (n >= 8) return *(const ds_u32x4 *)q;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) r[i / 2] |= (uint32_t)q[i] << (16 * (i % 2));
  return r;
}

// bring8's place in the tile for this thread, and where it goes in LDS ([kTile][kPitch]).
__device__ inline void place(bool k_last, int &p, int &k) {
  const int t = threadIdx.x;
  if (k_last) p = t / 4, k = t % 4 * 8;
  else p = t % 8 * 8, k = t / 8;
}
__device__ inline void put_in_lds(uint16_t *lds, bool k_last, u32x4 x) {
  int p, k;
  place(k_last, p, k);
  if (k_last) {
    *(u32x4 *)(lds + p * kPitch + k) = x;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) lds[(p + i) * kPitch + k] = (uint16_t)(x[i / 2] >> (16 * (i % 2)));
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void ds_matmul_kernel(Operand a, Operand b, Epilogue e, int64_t depth) {
  __shared__ union {
    struct {
      alignas(16) uint16_t a[kTile * kPitch], b[kTile * kPitch];
    } in;
    float out[kTile][kTile + 4];
  } lds;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t p0 = (int64_t)blockIdx.y * kTile, q0 = (int64_t)blockIdx.x * kTile;
  int pa, ka, pb, kb;
  place(a.k_last, pa, ka);
  place(b.k_last, pb, kb);
  f32x4 sum[4] = {};
  u32x4 na = {}, nb = {};
  if (depth > 0) na = bring8<T>(a, p0 + pa, ka, depth), nb = bring8<T>(b, q0 + pb, kb, depth);
  for (int64_t k = 0; k < depth; k += kDeep) {
    put_in_lds(lds.in.a, a.k_last, na);
    put_in_lds(lds.in.b, b.k_last, nb);
    __syncthreads();
    if (k + kDeep < depth) na = bring8<T>(a, p0 + pa, k + kDeep + ka, depth), nb = bring8<T>(b, q0 + pb, k + kDeep + kb, depth);
    const u32x4 x = *(const u32x4 *)(lds.in.a + (wave * 16 + lane % 16) * kPitch + lane / 16 * 8);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const u32x4 y = *(const u32x4 *)(lds.in.b + (t * 16 + lane % 16) * kPitch + lane / 16 * 8);
      sum[t] = mfma(y, x, sum[t], T());
    }
    __syncthreads();
  }
#pragma unroll
  for (int t = 0; t < 4; ++t) *(f32x4 *)&lds.out[wave * 16 + lane % 16][t * 16 + lane / 16 * 4] = sum[t];
  __syncthreads();
  for (int r = 0; r < 2; ++r) {
    const int row = r * 32 + threadIdx.x / 8, col = threadIdx.x % 8 * 8;
    const int64_t i = p0 + row, j = q0 + col, left = i < e.m ? e.n - j : 0;
    Eight z;
#pragma unroll
    for (int k = 0; k < 8; ++k) z.v[k] = lds.out[row][col + k];
    finish8(e, i, j, (int)(left < 0 ? 0 : left < 8 ? left : 8), z);
  }
}

// a (or b's transpose): p along `along` = its rows if `p_rows`.
Operand operand(const ds_matrix *m, bool p_rows) {
  const int64_t p = p_rows ? m->rows : m->cols, k = p_rows ? m->cols : m->rows;
  const int64_t step_p = p_rows ? m->row_stride : m->col_stride, step_k = p_rows ? m->col_stride : m->row_stride;
  // in rows if the columns are neighbours; a matrix of one row or column may be either
  const bool in_rows = (m->cols <= 1 || m->col_stride == 1) && (m->rows <= 1 || m->row_stride >= m->cols);
  const bool k_last = in_rows == p_rows;
  const int64_t ld = k_last ? (p > 1 ? step_p : k) : (k > 1 ? step_k : p);
  return Operand{m->base, ld, p, m->dtype == DS_MX8 ? m->scale : nullptr, m->scale_stride, k_last};
}

int check_product(const ds_matrix *a, const ds_matrix *b, const ds_matrix *c) {
  DS_TRY(ds_check_matrix(a, false));
  DS_TRY(ds_check_matrix(b, false));
  DS_TRY(ds_check_matrix(c, true));
  const bool a8 = a->dtype == DS_MX8, b8 = b->dtype == DS_MX8;
  if ((!a8 && !ds_is_half(a->dtype)) || (!b8 && !ds_is_half(b->dtype)) || (!a8 && !b8 && a->dtype != b->dtype) || c->dtype == DS_MX8 ||
      a->cols != b->rows || a->rows != c->rows || b->cols != c->cols)
    return DS_EINVAL;
  return DS_OK;
}

}  // namespace

extern "C" int ds_matmul_workspace(const ds_matrix *a, const ds_matrix *b, const ds_matrix *c, uint64_t *bytes) {
  if (!bytes) return DS_EINVAL;
  DS_TRY(check_product(a, b, c));
  *bytes = 0;
  return DS_OK;
}

extern "C" int ds_matmul(const ds_matrix *a, const ds_matrix *b, const ds_matrix *c, const ds_matmul_epilogue *epilogue, void *workspace,
                         uint64_t workspace_bytes, void *stream) {
  DS_TRY(check_product(a, b, c));
  static const ds_matmul_epilogue nothing = {nullptr, DS_F32, DS_ACT_NONE, nullptr, nullptr};
  const ds_matmul_epilogue &ep = epilogue ? *epilogue : nothing;
  if (ep.act > DS_ACT_SILU || (ep.bias && (!ds_is_float(ep.bias_dtype) || ds_misaligned(ep.bias, ds_itemsize(ep.bias_dtype))))) return DS_EINVAL;
  if (ep.residual) {
    DS_TRY(ds_check_matrix(ep.residual, true));
    if (ep.residual->dtype != c->dtype || !ds_same_extents(ep.residual, c)) return DS_EINVAL;
  }
  if (ep.saved) {
    DS_TRY(ds_check_matrix(ep.saved, true));
    if (ep.saved->dtype != DS_MX8 || !ds_same_extents(ep.saved, c)) return DS_EINVAL;
  }
  if (c->rows == 0 || c->cols == 0) return DS_OK;
  (void)workspace, (void)workspace_bytes;
  const Operand oa = operand(a, true), ob = operand(b, false);
  const Epilogue e{ds_rows(c), ds_rows(ep.residual), ds_rows(ep.saved), ep.bias, c->rows, c->cols, c->dtype, ep.bias_dtype, ep.act};
  const dim3 grid((uint32_t)((c->cols + kTile - 1) / kTile), (uint32_t)((c->rows + kTile - 1) / kTile));
  if (grid.y > 65535) return DS_ERANGE;
  hipStream_t st = (hipStream_t)stream;
  if (a->dtype == DS_F16 || b->dtype == DS_F16)
    hipLaunchKernelGGL(ds_matmul_kernel<__half>, grid, dim3(kThreads), 0, st, oa, ob, e, a->cols);
  else
    hipLaunchKernelGGL(ds_matmul_kernel<__hip_bfloat16>, grid, dim3(kThreads), 0, st, oa, ob, e, a->cols);
  DS_HIP_TRY(hipGetLastError());
  return DS_OK;
}
