// Layer norm, forward and backward.
//
// Both are bound by HBM: every element is read once and written once.  A row belongs to a wavefront or to a work-group, whose
// threads hold it in registers, in pieces of eight neighbouring columns; the mean is taken first and the squares of the
// differences from it then, out of the registers, so that a row whose mean is large beside its spread keeps its variance.  A
// work-group walks over several rows, with gamma and beta in registers, and asks for the next row's data before it computes on
// this one's.  Backward, a thread also sums its columns' share of dgamma and dbeta over its rows; those sums are a line of `partial`
// for each work-group, and a second launch adds the lines in their order.  Rows too long for the registers are read again for
// every pass, out of the caches.
//
// 8192 rows of 4096 bfloat16: forward with a checkpoint in 8 bits 34 us (168 MB, 4.9 TB/s), backward from it with a residual 49 us (236
// MB, 4.8 TB/s) and 6 us for the lines.  One row of 8192: 4 us, the chain of its loads, two sums over 16 wavefronts and the store.

#include <type_traits>

#include "ds_ops.h"

namespace {

// The sum of `x` over the `WAVES` wavefronts of a row, in every thread.  `room`: one float per wavefront; two such rooms are used
// in turn, so that one barrier is enough: a wavefront writes to a room again only behind the barrier of the other.
template <int WAVES>
__device__ inline float row_sum(float x, float *room) {
  x = wave_sum(x);
  if (WAVES == 1) return x;
  if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = x;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) s += room[w];
  return s;
}

__device__ inline int columns_left(int64_t cols, int64_t j) {
  const int64_t left = cols - j;
  return (int)(left < 0 ? 0 : left < 8 ? left : 8);
}

// The compiler is not to keep what it has computed from these bits.
template <typename B>
__device__ inline void opaque(B &bits) {
  uint32_t *w = (uint32_t *)&bits;
#pragma unroll
  for (int k = 0; k < (int)sizeof(B) / 4; ++k) asm volatile("" : "+v"(w[k]));
}

struct NormForward {
  Rows x, y, saved;
  const void *gamma, *beta;
  float *mean, *rstd;
  int64_t rows, cols;
  float eps;
  uint32_t param_dtype;
};

// What a row's mean and rstd are kept and used as.
__device__ inline void put_statistics(const NormForward &a, int64_t i, float mean, float rstd) {
  if (a.mean) a.mean[i] = mean;
  if (a.rstd) a.rstd[i] = rstd;
}

// WAVES wavefronts have a row, each thread HAS pieces of eight columns, 512 * WAVES apart; a work-group of WIDE wavefronts has
// WIDE / WAVES rows at a time.
template <typename T, int WAVES, int WIDE, int HAS>
__global__ __launch_bounds__(WIDE * 64) void ds_layernorm_forward_kernel(NormForward a) {
  __shared__ float room[2][WIDE];
  constexpr int kRows = WIDE / WAVES, kApart = WAVES * 512;
  const int at = threadIdx.x % (WAVES * 64) * 8, which = threadIdx.x / (WAVES * 64);
  Eight g[HAS], b[HAS];
  int n[HAS];
  const float each = 1.f / (float)a.cols;
  const int64_t stride = (int64_t)gridDim.x * kRows;
  int64_t i = (int64_t)blockIdx.x * kRows + which;
  typename RowsOf<T>::Bits next[HAS];
  AnyBits gamma[HAS], beta[HAS];
#pragma unroll
  for (int p = 0; p < HAS; ++p) {
    const int64_t j = at + p * kApart;
    n[p] = columns_left(a.cols, j);
    next[p] = RowsOf<T>::ask(a.x, i, j, i < a.rows ? n[p] : 0);
    gamma[p] = ask_up_to8_any(a.gamma, a.param_dtype, j, n[p]), beta[p] = ask_up_to8_any(a.beta, a.param_dtype, j, n[p]);
  }
#pragma unroll
  for (int p = 0; p < HAS; ++p) g[p] = value_any(gamma[p], a.gamma, a.param_dtype, 1.f), b[p] = value_any(beta[p], a.beta, a.param_dtype, 0.f);
  for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.rows; first += stride, i += stride) {
    Eight x[HAS];
    float sum = 0.f, squares = 0.f;
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
      x[p] = RowsOf<T>::value(next[p], n[p]);
#pragma unroll
      for (int k = 0; k < 8; ++k) sum += x[p].v[k];
    }
#pragma unroll
    for (int p = 0; p < HAS; ++p) next[p] = RowsOf<T>::ask(a.x, i + stride, at + p * kApart, i + stride < a.rows ? n[p] : 0);
    const float mean = row_sum<WAVES>(sum, room[0]) * each;
    const bool row = i < a.rows;
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
      if (a.saved.base) mx8_put(a.saved, i, at + p * kApart, row ? n[p] : 0, x[p]);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[p].v[k] -= mean;
        squares += k < n[p] ? x[p].v[k] * x[p].v[k] : 0.f;
      }
    }
    const float rstd = 1.f / sqrtf(row_sum<WAVES>(squares, room[1]) * each + a.eps);
    if (!row) continue;
    if (at == 0) put_statistics(a, i, mean, rstd);
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[p].v[k] = x[p].v[k] * rstd * g[p].v[k] + b[p].v[k];
      put_up_to8<T>(a.y.base, i * a.y.stride + at + p * kApart, n[p], x[p]);
    }
  }
}

// Rows of any length.
template <typename T>
__global__ __launch_bounds__(1024) void ds_layernorm_forward_long_kernel(NormForward a) {
  __shared__ float room[2][16];
  constexpr int kApart = 1024 * 8;
  const float each = 1.f / (float)a.cols;
  for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x) {
    float sum = 0.f, squares = 0.f;
    for (int64_t j = threadIdx.x * 8; j < a.cols; j += kApart) {
      const Eight x = RowsOf<T>::get(a.x, i, j, columns_left(a.cols, j));
#pragma unroll
      for (int k = 0; k < 8; ++k) sum += x.v[k];
    }
    const float mean = row_sum<16>(sum, room[0]) * each;
    for (int64_t j = threadIdx.x * 8; j < a.cols; j += kApart) {
      const int n = columns_left(a.cols, j);
      const Eight x = RowsOf<T>::get(a.x, i, j, n);
#pragma unroll
      for (int k = 0; k < 8; ++k) squares += k < n ? (x.v[k] - mean) * (x.v[k] - mean) : 0.f;
    }
    const float rstd = 1.f / sqrtf(row_sum<16>(squares, room[1]) * each + a.eps);
    if (threadIdx.x == 0) put_statistics(a, i, mean, rstd);
    for (int64_t first = 0; first < a.cols; first += kApart) {
      const int64_t j = first + threadIdx.x * 8;
      const int n = columns_left(a.cols, j);
      Eight x = RowsOf<T>::get(a.x, i, j, n);
      if (a.saved.base) mx8_put(a.saved, i, j, n, x);
      const Eight g = get_up_to8_any(a.gamma, a.param_dtype, j, n, 1.f), b = get_up_to8_any(a.beta, a.param_dtype, j, n, 0.f);
#pragma unroll
      for (int k = 0; k < 8; ++k) x.v[k] = (x.v[k] - mean) * rstd * g.v[k] + b.v[k];
      put_up_to8<T>(a.y.base, i * a.y.stride + j, n, x);
    }
  }
}

struct NormBackward {
  Rows dy, x, residual, dx;
  const float *mean, *rstd;
  const void *gamma;
  float *partial;  // [2][parts][cols]: dgamma's lines, then dbeta's; or NULL
  int64_t rows, cols;
  uint32_t param_dtype;
};

// dx, and the sums of the work-group's rows.  The shapes are the forward kernel's.
template <typename T, typename X, int WAVES, int WIDE, int HAS>
__global__ __launch_bounds__(WIDE * 64) void ds_layernorm_backward_kernel(NormBackward a) {
  constexpr int kRows = WIDE / WAVES, kApart = WAVES * 512;
  __shared__ float room[2][2][WIDE];
  __shared__ float lines[kRows > 1 ? kRows : 1][kRows > 1 ? HAS * kApart : 1];
  const int at = threadIdx.x % (WAVES * 64) * 8, which = threadIdx.x / (WAVES * 64);
  Eight g[HAS], dg[HAS] = {}, db[HAS] = {};
  int n[HAS];
  AnyBits gamma[HAS];
#pragma unroll
  for (int p = 0; p < HAS; ++p) {
    n[p] = columns_left(a.cols, at + p * kApart);
    gamma[p] = ask_up_to8_any(a.gamma, a.param_dtype, at + p * kApart, n[p]);
  }
  const float each = 1.f / (float)a.cols;
  const int64_t stride = (int64_t)gridDim.x * kRows;
  int64_t i = (int64_t)blockIdx.x * kRows + which;
  struct Row {
    typename RowsOf<T>::Bits d[HAS], r[HAS];
    typename RowsOf<X>::Bits x[HAS];
    float mean, rstd;
  };
  const auto ask = [&](Row &o, int64_t i) {
    const bool row = i < a.rows;
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
      const int64_t j = at + p * kApart;
      o.d[p] = RowsOf<T>::ask(a.dy, i, j, row ? n[p] : 0);
      o.x[p] = RowsOf<X>::ask(a.x, i, j, row ? n[p] : 0);
      if (a.residual.base) o.r[p] = RowsOf<T>::ask(a.residual, i, j, row ? n[p] : 0);
    }
    o.mean = row ? a.mean[i] : 0.f, o.rstd = row ? a.rstd[i] : 0.f;
  };
  Row next = {};
  ask(next, i);
#pragma unroll
  for (int p = 0; p < HAS; ++p) g[p] = value_any(gamma[p], a.gamma, a.param_dtype, 1.f);
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.rows; first += stride, i += stride, turn ^= 1) {
    Row now = next;
    float flat = 0.f, along = 0.f;
    // h and dy are computed once more for dx, from the bits, which are a third of the registers.  (Beyond the row dy is 0, and h
    // finite where the row's is.)
    const auto terms = [&](int p, Eight &d, Eight &h) {
      h = RowsOf<X>::value(now.x[p], 8), d = RowsOf<T>::value(now.d[p], 8);
#pragma unroll
      for (int k = 0; k < 8; ++k) h.v[k] = (h.v[k] - now.mean) * now.rstd;
    };
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
      Eight d, h;
      terms(p, d, h);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float w = d.v[k] * g[p].v[k];
        db[p].v[k] += d.v[k];
        dg[p].v[k] += d.v[k] * h.v[k];
        flat += w;
        along += w * h.v[k];
      }
    }
    ask(next, i + stride);
    if (WAVES == 1) {
      flat = wave_sum(flat) * each, along = wave_sum(along) * each;
    } else {
      flat = wave_sum(flat), along = wave_sum(along);
      if ((threadIdx.x & 63) == 0) room[turn][0][threadIdx.x >> 6] = flat, room[turn][1][threadIdx.x >> 6] = along;
      __syncthreads();
      flat = along = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) flat += room[turn][0][w], along += room[turn][1][w];
      flat *= each, along *= each;
    }
    if (i >= a.rows) continue;
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
      opaque(now.x[p]), opaque(now.d[p]);
      Eight out = {}, d, h;
      terms(p, d, h);
      if (a.residual.base) out = RowsOf<T>::value(now.r[p], 8);
#pragma unroll
      for (int k = 0; k < 8; ++k) out.v[k] += now.rstd * (d.v[k] * g[p].v[k] - flat - h.v[k] * along);
      put_up_to8<T>(a.dx.base, i * a.dx.stride + at + p * kApart, n[p], out);
    }
  }
  if (!a.partial) return;
  const int64_t parts = gridDim.x;
  if (kRows == 1) {
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
      const int64_t j = at + p * kApart;
      put_up_to8<float>(a.partial, blockIdx.x * a.cols + j, n[p], dg[p]);
      put_up_to8<float>(a.partial, (parts + blockIdx.x) * a.cols + j, n[p], db[p]);
    }
    return;
  }
  // the rows' wavefronts are added in their order
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    __syncthreads();
#pragma unroll
    for (int p = 0; p < HAS; ++p)
#pragma unroll
      for (int k = 0; k < 8; ++k) lines[which][at + p * kApart + k] = s ? db[p].v[k] : dg[p].v[k];
    __syncthreads();
    for (int j = threadIdx.x; j < a.cols; j += WIDE * 64) {
      float sum = 0.f;
#pragma unroll
      for (int r = 0; r < kRows; ++r) sum += lines[r][j];
      a.partial[(s * parts + blockIdx.x) * a.cols + j] = sum;
    }
  }
}

// Rows of any length: a row's sums and dx.
template <typename T, typename X>
__global__ __launch_bounds__(1024) void ds_layernorm_backward_long_kernel(NormBackward a) {
  __shared__ float room[2][16];
  constexpr int kApart = 1024 * 8;
  const float each = 1.f / (float)a.cols;
  for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x) {
    const float mean = a.mean[i], rstd = a.rstd[i];
    float flat = 0.f, along = 0.f;
    for (int64_t j = threadIdx.x * 8; j < a.cols; j += kApart) {
      const int n = columns_left(a.cols, j);
      const Eight d = RowsOf<T>::get(a.dy, i, j, n), x = RowsOf<X>::get(a.x, i, j, n), g = get_up_to8_any(a.gamma, a.param_dtype, j, n, 1.f);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float w = d.v[k] * g.v[k];
        flat += w;
        along += k < n ? w * ((x.v[k] - mean) * rstd) : 0.f;
      }
    }
    flat = row_sum<16>(flat, room[0]) * each;
    along = row_sum<16>(along, room[1]) * each;
    for (int64_t j = threadIdx.x * 8; j < a.cols; j += kApart) {
      const int n = columns_left(a.cols, j);
      const Eight d = RowsOf<T>::get(a.dy, i, j, n), x = RowsOf<X>::get(a.x, i, j, n), g = get_up_to8_any(a.gamma, a.param_dtype, j, n, 1.f);
      Eight r = {};
      if (a.residual.base) r = RowsOf<T>::get(a.residual, i, j, n);
#pragma unroll
      for (int k = 0; k < 8; ++k) r.v[k] += rstd * (d.v[k] * g.v[k] - flat - (x.v[k] - mean) * rstd * along);
      put_up_to8<T>(a.dx.base, i * a.dx.stride + j, n, r);
    }
  }
}

// Rows of any length: the lines of dgamma and dbeta.  A work-group has 512 columns and every (4 * parts)-th row for each of its
// wavefronts.
template <typename T, typename X>
__global__ __launch_bounds__(256) void ds_layernorm_params_long_kernel(NormBackward a) {
  __shared__ float sums[2][4][64][8 + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t j = ((int64_t)blockIdx.x * 64 + lane) * 8;
  const int n = columns_left(a.cols, j);
  Eight dg = {}, db = {};
  for (int64_t i = (int64_t)blockIdx.y * 4 + wave; i < a.rows; i += (int64_t)gridDim.y * 4) {
    const float mean = a.mean[i], rstd = a.rstd[i];
    const Eight d = RowsOf<T>::get(a.dy, i, j, n), x = RowsOf<X>::get(a.x, i, j, n);
#pragma unroll
    for (int k = 0; k < 8; ++k) dg.v[k] += k < n ? d.v[k] * ((x.v[k] - mean) * rstd) : 0.f, db.v[k] += d.v[k];
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) sums[0][wave][lane][k] = dg.v[k], sums[1][wave][lane][k] = db.v[k];
  __syncthreads();
  for (int c = threadIdx.x; c < 1024; c += 256) {
    const int which = c / 512, at = c % 512;
    const int64_t col = (int64_t)blockIdx.x * 512 + at;
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) s += sums[which][w][at / 8][at % 8];
    if (col < a.cols) a.partial[((int64_t)which * gridDim.y + blockIdx.y) * a.cols + col] = s;
  }
}

// Rows of so many columns fit the registers of a work-group with two pieces a thread: forward of 16 wavefronts, backward of 8 (with two
// pieces a thread has about 200 registers, and 16 wavefronts leave each thread 128; one piece on 16 is not tried).
constexpr int64_t kLongest = 16384, kLongestBackward = 8192;

// Work-groups: as many as run at once, or one for each set of rows.  (Backward each is a line that is written and read again.)
int64_t norm_groups(int64_t rows, int64_t at_a_time, int64_t most) {
  const int64_t sets = (rows + at_a_time - 1) / at_a_time;
  return sets < most ? sets : most;
}

template <typename T>
int launch_forward(const NormForward &a, hipStream_t stream) {
  const auto launch = [&](auto kernel, int rows, int waves) -> int {
    hipLaunchKernelGGL(kernel, dim3((uint32_t)norm_groups(a.rows, rows, 256 * 32 / waves)), dim3(waves * 64), 0, stream, a);
    DS_HIP_TRY(hipGetLastError());
    return DS_OK;
  };
  // few rows: as many wavefronts for each as have something to read
  if (a.rows <= 256 && a.cols > 512 && a.cols <= 8192) {
    if (a.cols <= 2048) return launch(ds_layernorm_forward_kernel<T, 4, 4, 1>, 1, 4);
    return launch(ds_layernorm_forward_kernel<T, 16, 16, 1>, 1, 16);
  }
  if (a.cols <= 512) return launch(ds_layernorm_forward_kernel<T, 1, 4, 1>, 4, 4);
  if (a.cols <= 1024) return launch(ds_layernorm_forward_kernel<T, 1, 4, 2>, 4, 4);
  if (a.cols <= 2048) return launch(ds_layernorm_forward_kernel<T, 4, 4, 1>, 1, 4);
  if (a.cols <= 4096) return launch(ds_layernorm_forward_kernel<T, 4, 4, 2>, 1, 4);
  if (a.cols <= 8192) return launch(ds_layernorm_forward_kernel<T, 8, 8, 2>, 1, 8);
  if (a.cols <= kLongest) return launch(ds_layernorm_forward_kernel<T, 16, 16, 2>, 1, 16);
  return launch(ds_layernorm_forward_long_kernel<T>, 1, 16);
}

int64_t norm_parts(int64_t rows, int64_t cols) {
  if (rows <= 0) return 1;
  if (cols <= 1024) return norm_groups(rows, 4, 512);
  if (cols <= kLongestBackward) return norm_groups(rows, 1, 512);
  const int64_t across = (cols + 511) / 512;
  return norm_groups(rows, 4, (1024 + across - 1) / across);
}

template <typename T, typename X>
int launch_backward(const NormBackward &a, int64_t parts, hipStream_t stream) {
  const auto launch = [&](auto kernel, int waves) -> int {
    hipLaunchKernelGGL(kernel, dim3((uint32_t)parts), dim3(waves * 64), 0, stream, a);
    DS_HIP_TRY(hipGetLastError());
    return DS_OK;
  };
  if (a.cols <= 512) return launch(ds_layernorm_backward_kernel<T, X, 1, 4, 1>, 4);
  if (a.cols <= 1024) return launch(ds_layernorm_backward_kernel<T, X, 1, 4, 2>, 4);
  if (a.cols <= 2048) return launch(ds_layernorm_backward_kernel<T, X, 4, 4, 1>, 4);
  if (a.cols <= 4096) return launch(ds_layernorm_backward_kernel<T, X, 4, 4, 2>, 4);
  if (a.cols <= kLongestBackward) return launch(ds_layernorm_backward_kernel<T, X, 8, 8, 2>, 8);
  // the parameters' sums first: dx may be dy
  if (a.partial) {
    hipLaunchKernelGGL((ds_layernorm_params_long_kernel<T, X>), dim3((uint32_t)((a.cols + 511) / 512), (uint32_t)parts), dim3(256), 0, stream, a);
    DS_HIP_TRY(hipGetLastError());
  }
  hipLaunchKernelGGL((ds_layernorm_backward_long_kernel<T, X>), dim3((uint32_t)norm_groups(a.rows, 1, 4096)), dim3(1024), 0, stream, a);
  DS_HIP_TRY(hipGetLastError());
  return DS_OK;
}

}  // namespace

extern "C" int ds_layernorm_forward(const ds_matrix *x, const void *gamma, const void *beta, uint32_t param_dtype, float eps,
                                    const ds_matrix *y, float *mean, float *rstd, const ds_matrix *saved, void *stream) {
  DS_TRY(ds_check_matrix(x, true));
  DS_TRY(ds_check_matrix(y, true));
  if (saved) DS_TRY(ds_check_matrix(saved, true));
  if (x->dtype == DS_MX8 || y->dtype != x->dtype || !ds_same_extents(x, y) || !ds_is_float(param_dtype) || !(eps >= 0.f) ||
      (saved && (saved->dtype != DS_MX8 || !ds_same_extents(x, saved))) || ds_misaligned(mean, 4) || ds_misaligned(rstd, 4) ||
      ds_misaligned(gamma, ds_itemsize(param_dtype)) || ds_misaligned(beta, ds_itemsize(param_dtype)))
    return DS_EINVAL;
  if (x->rows == 0 || x->cols == 0) return DS_OK;
  const NormForward a{ds_rows(x), ds_rows(y), ds_rows(saved), gamma, beta, mean, rstd, x->rows, x->cols, eps, param_dtype};
  return ds_with_type(x->dtype, [&](auto type) -> int {
    typedef decltype(type) T;
    return launch_forward<T>(a, (hipStream_t)stream);
  });
}

extern "C" int ds_layernorm_backward_workspace(int64_t rows, int64_t cols, uint64_t *bytes) {
  if (!bytes || rows < 0 || cols < 0) return DS_EINVAL;
  if (rows > kMaxExtent || cols > kMaxExtent) return DS_ERANGE;
  *bytes = (uint64_t)(2 * norm_parts(rows, cols) * cols * 4);
  return DS_OK;
}

extern "C" int ds_layernorm_backward(const ds_matrix *dy, const ds_matrix *x, const float *mean, const float *rstd, const void *gamma,
                                     uint32_t param_dtype, const ds_matrix *residual, const ds_matrix *dx, float *dgamma, float *dbeta,
                                     void *workspace, uint64_t workspace_bytes, void *stream) {
  DS_TRY(ds_check_matrix(dy, true));
  DS_TRY(ds_check_matrix(x, true));
  DS_TRY(ds_check_matrix(dx, true));
  if (residual) DS_TRY(ds_check_matrix(residual, true));
  const int64_t rows = dy->rows, cols = dy->cols;
  if (dy->dtype == DS_MX8 || dx->dtype != dy->dtype || (x->dtype != DS_MX8 && x->dtype != dy->dtype) || !ds_same_extents(dy, x) ||
      !ds_same_extents(dy, dx) || (residual && (residual->dtype != dy->dtype || !ds_same_extents(dy, residual))) ||
      !ds_is_float(param_dtype) || ds_misaligned(gamma, ds_itemsize(param_dtype)) || ds_misaligned(mean, 4) || ds_misaligned(rstd, 4) ||
      ds_misaligned(dgamma, 4) || ds_misaligned(dbeta, 4))
    return DS_EINVAL;
  const bool sums = dgamma || dbeta;
  if (cols == 0 || (rows == 0 && !sums)) return DS_OK;
  if (rows > 0 && (!mean || !rstd)) return DS_EINVAL;
  const int64_t parts = norm_parts(rows, cols);
  if (sums) {
    if (!workspace || ds_misaligned(workspace, 16)) return DS_EINVAL;
    if (workspace_bytes < (uint64_t)(2 * parts * cols * 4)) return DS_ERANGE;
  }
  hipStream_t st = (hipStream_t)stream;
  const NormBackward a{ds_rows(dy), ds_rows(x), ds_rows(residual), ds_rows(dx), mean, rstd, gamma, sums ? (float *)workspace : nullptr, rows, cols, param_dtype};
  if (rows > 0)
    DS_TRY(ds_with_type(dy->dtype, [&](auto type) -> int {
      typedef decltype(type) T;
      return x->dtype == DS_MX8 ? launch_backward<T, Mx8>(a, parts, st) : launch_backward<T, T>(a, parts, st);
    }));
  const int64_t lines = rows > 0 ? parts : 0;
  if (!sums) return DS_OK;
  return ds_launch_sum_parts((const float *)workspace, lines, cols, dgamma, dbeta, st);
}
