// AdamW over the tensors of a table, and the sum of the squares of their gradients.
//
// Both are bound by HBM.  The table cuts every tensor into chunks of kPieces pieces of eight neighbouring columns; a work-group
// takes a chunk, and each of its threads kEach pieces, 256 apart, whose data are all on their way before the first is computed on.
// Moments in 8 bits are in groups of 32 columns, which four neighbouring lanes hold, as everywhere in this library.  What the
// table's tensors have in common (types, kind of moments) is a kernel's template, and a launch has the chunks of one kind.
//
// What all elements share -- 1 - beta^t, the factor of clipping -- is computed from device memory, so that a captured graph
// takes another step whenever it is replayed: by the first wavefront of every work-group, in 64 bits, while the data come.

#include <algorithm>
#include <cmath>
#include <new>
#include <type_traits>
#include <utility>
#include <vector>

#include "ds_ops.h"

namespace {

constexpr int kThreads = 256;
constexpr int kEach = 2;                     // pieces of a thread
constexpr int64_t kPieces = kThreads * kEach;  // of a chunk
constexpr int64_t kSquareGroups = 2048;      // work-groups of the sum of squares, for each kind of tensors

// A tensor in the table.  Its matrices are one row where that is how they lie.
struct Tensor {
  Rows param, grad, m, v, copy;
  int64_t rows, cols, pieces;  // pieces of a row: a multiple of four where moments have 8 bits
  uint32_t number, copy_dtype;
  float decay, rate;
};
struct Chunk {
  int64_t piece;  // the first one
  uint32_t tensor, reserved;
};
// A kind of tensors: their types, and their chunks.
struct Kind {
  uint32_t param, grad, eight;
  int64_t begin, end;
};

struct Settings {
  double rate, log_beta1, log_beta2, grad_scale, most_norm;
  const int64_t *step;
  const float *rate_now;
  const double *squares;
  float beta1, beta2, rest1, rest2, eps;
  uint32_t seed;  // both halves mixed
};

__host__ __device__ inline uint32_t mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x9E3779B9u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ x >> 16;
}

struct Now {
  float rate;      // settings'
  float step;      // 1 / (1 - beta1^t)
  float root;      // 1 / sqrt(1 - beta2^t)
  float grad;      // what a gradient is multiplied with
  uint32_t key;    // mix(t + mix(seed))
  uint32_t still;  // nothing is to change
};

__device__ inline Now now_of(const Settings &s) {
  Now w;
  const int64_t at = *s.step, t = at < 1 ? 1 : at;
  w.rate = s.rate_now ? *s.rate_now : (float)s.rate;
  w.key = mix((uint32_t)t + s.seed);
  w.step = (float)(-1.0 / expm1((double)t * s.log_beta1));
  w.root = (float)(1.0 / sqrt(-expm1((double)t * s.log_beta2)));
  w.still = 0;
  double c = s.grad_scale;
  if (s.squares) {
    const double sum = *s.squares, norm = sqrt(sum) * fabs(s.grad_scale);
    w.still = !(sum < (double)INFINITY);
    if (s.most_norm > 0.0 && norm > s.most_norm) c = c * s.most_norm / norm;
  }
  w.grad = (float)c;
  return w;
}

// Where piece `item` of a tensor is: its row, its first column, and how many columns of it are there.
__device__ inline void place_of(const Tensor &t, int64_t item, int64_t &i, int64_t &j, int &n) {
  if (t.rows == 1) i = 0, j = item;
  else if (t.rows * t.pieces <= 0xffffffffll - kPieces) i = (uint32_t)item / (uint32_t)t.pieces, j = (uint32_t)item - (uint32_t)i * (uint32_t)t.pieces;
  else i = item / t.pieces, j = item - i * t.pieces;
  j *= 8;
  const int64_t left = i < t.rows ? t.cols - j : 0;
  n = (int)(left < 0 ? 0 : left < 8 ? left : 8);
}

__device__ inline void put_copy(const Tensor &t, int64_t i, int64_t j, int n, const Eight &p) {
  const int64_t at = i * t.copy.stride + j;
  if (t.copy_dtype == DS_BF16) put_up_to8<__hip_bfloat16>(t.copy.base, at, n, p);
  else if (t.copy_dtype == DS_F16) put_up_to8<__half>(t.copy.base, at, n, p);
  else put_up_to8<float>(t.copy.base, at, n, p);
}

template <typename P, typename G, bool EIGHT>
__global__ __launch_bounds__(kThreads) void ds_adamw_step_kernel(const Tensor *tensors, const Chunk *chunks, int64_t count, Settings s) {
  typedef std::conditional_t<EIGHT, Mx8, float> M;
  typedef std::conditional_t<EIGHT, Uf8, float> V;
  __shared__ Now shared;
  for (int64_t c = blockIdx.x; c < count; c += gridDim.x) {
    const Chunk chunk = chunks[c];
    const Tensor t = tensors[chunk.tensor];
    int64_t i[kEach], j[kEach];
    int n[kEach];
    typename RowsOf<P>::Bits p[kEach];
    typename RowsOf<G>::Bits g[kEach];
    typename RowsOf<M>::Bits m[kEach];
    typename RowsOf<V>::Bits v[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      place_of(t, chunk.piece + e * kThreads + threadIdx.x, i[e], j[e], n[e]);
      p[e] = RowsOf<P>::ask(t.param, i[e], j[e], n[e]), g[e] = RowsOf<G>::ask(t.grad, i[e], j[e], n[e]);
      m[e] = RowsOf<M>::ask(t.m, i[e], j[e], n[e]), v[e] = RowsOf<V>::ask(t.v, i[e], j[e], n[e]);
    }
    if (c == blockIdx.x) {
      if (threadIdx.x < 64) {
        const Now w = now_of(s);
        if (threadIdx.x == 0) shared = w;
      }
      __syncthreads();
    }
    const Now w = shared;
    if (w.still) return;
    const float rate = w.rate * t.rate, step = rate * w.step, decay = rate * t.decay;
    const uint32_t key = mix(t.number + w.key);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      Eight param = RowsOf<P>::value(p[e], n[e]), first = RowsOf<M>::value(m[e], n[e]), second = RowsOf<V>::value(v[e], n[e]);
      const Eight grad = RowsOf<G>::value(g[e], n[e]);
      {
        // rounded after each operation, so that a code, which the last bit may decide, is what the formula in 32 bits says anywhere
#pragma clang fp contract(off)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float x = grad.v[k] * w.grad;
          first.v[k] = first.v[k] * s.beta1 + x * s.rest1;
          second.v[k] = second.v[k] * s.beta2 + x * x * s.rest2;
        }
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        param.v[k] -= decay * param.v[k] + step * first.v[k] / (sqrtf(second.v[k]) * w.root + s.eps);
      }
      put_up_to8<P>(t.param.base, i[e] * t.param.stride + j[e], n[e], param);
      if (t.copy.base) put_copy(t, i[e], j[e], n[e], param);
      if constexpr (EIGHT) {
        const uint32_t at = (uint32_t)(i[e] * t.cols + j[e]) + key;
        const uint32_t scale_m = mx8_scale(max_of_four_lanes(magnitude8(first)));
        const uint32_t scale_v = uf8_scale(max_of_four_lanes(largest_bits8(second)));
        ds_u32x2 code_m = {0, 0}, code_v = {0, 0};
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t r = mix(at + k);
          const float u = ((float)(r & 0xffffu) + 0.5f) * 0x1p-16f;
          const float q = __builtin_floorf(ldexpf(first.v[k], 133 - (int)scale_m) + u);
          const uint32_t byte = (uint32_t)(int)__builtin_amdgcn_fmed3f(q, -127.f, 127.f) & 255u;
          code_m[k / 4] |= (scale_m == 0u || scale_m == 255u ? 0u : byte) << (8 * (k % 4));
          code_v[k / 4] |= uf8_code(__float_as_uint(second.v[k]), (r >> 16 << 4) + 8u, scale_v) << (8 * (k % 4));
        }
        eight_put(t.m, i[e], j[e], n[e], code_m, scale_m);
        eight_put(t.v, i[e], j[e], n[e], code_v, scale_v);
      } else {
        put_up_to8<float>(t.m.base, i[e] * t.m.stride + j[e], n[e], first);
        put_up_to8<float>(t.v.base, i[e] * t.v.stride + j[e], n[e], second);
      }
    }
  }
}

__device__ inline double wave_sum(double x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d, 64);
  return x;
}

// One sum for each work-group, in the order of its chunks.  (In 64 bits: gradients' squares span more than 32 bits' exponents do, and
// the sums of ranks are added.)
template <typename G>
__global__ __launch_bounds__(kThreads) void ds_adamw_squares_kernel(const Tensor *tensors, const Chunk *chunks, int64_t count, double *partial) {
  __shared__ double sums[kThreads / 64];
  double sum = 0.0;
  for (int64_t c = blockIdx.x; c < count; c += gridDim.x) {
    const Chunk chunk = chunks[c];
    const Tensor &t = tensors[chunk.tensor];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      int64_t i, j;
      int n;
      place_of(t, chunk.piece + e * kThreads + threadIdx.x, i, j, n);
      const Eight g = RowsOf<G>::get(t.grad, i, j, n);
#pragma unroll
      for (int k = 0; k < 8; ++k) sum += (double)g.v[k] * (double)g.v[k];
    }
  }
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) partial[blockIdx.x] = sums[0] + sums[1] + (sums[2] + sums[3]);
}

__global__ __launch_bounds__(1024) void ds_adamw_squares_sum_kernel(const double *partial, int64_t count, double *squares) {
  __shared__ double sums[16];
  double sum = 0.0;
  for (int64_t k = threadIdx.x; k < count; k += 1024) sum += partial[k];
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x) return;
  sum = 0.0;
  for (int w = 0; w < 16; ++w) sum += sums[w];
  *squares = sum;
}

int64_t square_groups(const Kind &k) { return std::min(k.end - k.begin, kSquareGroups); }

// Memory that a step writes.
struct Range {
  uintptr_t begin, end;
  bool whole;  // all of it is written
};

void add_range(std::vector<Range> &ranges, const void *base, int64_t rows, int64_t cols, int64_t stride, int64_t size) {
  if (!base) return;
  const uintptr_t from = (uintptr_t)base, past = from + (uintptr_t)(((rows > 1 ? stride * (rows - 1) : 0) + cols) * size);
  ranges.push_back({from, past, rows == 1 || stride == cols});
}

bool written_twice(std::vector<Range> &ranges) {
  std::sort(ranges.begin(), ranges.end(), [](const Range &a, const Range &b) { return a.begin < b.begin; });
  uintptr_t covered = 0;  // the end of the whole ranges so far
  for (size_t k = 0; k < ranges.size(); ++k) {
    const Range &r = ranges[k];
    if (k && ranges[k - 1].begin == r.begin) return true;
    if (!r.whole) continue;
    if (r.begin < covered) return true;
    covered = std::max(covered, r.end);
  }
  return false;
}

}  // namespace

struct ds_adamw {
  int device = -1;
  void *memory = nullptr;
  const Tensor *tensors = nullptr;
  const Chunk *chunks = nullptr;
  std::vector<Kind> kinds;
  int64_t parts() const {
    int64_t sum = 0;
    for (const Kind &k : kinds) sum += square_groups(k);
    return sum;
  }
};

namespace {

int check_tensor(const ds_adamw_tensor &t, bool &copied) {
  const auto is = [&](const ds_matrix &m) -> int {
    DS_TRY(ds_check_matrix(&m, true));
    return m.dtype != DS_MX8 && ds_same_extents(&t.param, &m) ? DS_OK : DS_EINVAL;
  };
  DS_TRY(is(t.param));
  DS_TRY(is(t.grad));
  if (t.m.dtype == DS_MX8) {
    DS_TRY(ds_check_matrix(&t.m, true));
    DS_TRY(ds_check_uf8(&t.v));
    if (!ds_same_extents(&t.param, &t.m) || !ds_same_extents(&t.param, &t.v)) return DS_EINVAL;
  } else {
    DS_TRY(is(t.m));
    DS_TRY(is(t.v));
    if (t.m.dtype != DS_F32 || t.v.dtype != DS_F32) return DS_EINVAL;
  }
  const ds_matrix &c = t.copy;
  copied = c.base || c.rows || c.cols || c.row_stride || c.col_stride || c.scale || c.scale_stride || c.reserved;
  if (copied) DS_TRY(is(c));
  return t.decay >= 0.f && t.decay < INFINITY && t.rate >= 0.f && t.rate < INFINITY ? DS_OK : DS_EINVAL;
}

// Does a matrix lie as one row?
bool one_row(const ds_matrix &m, bool eight) {
  return m.rows <= 1 || (m.row_stride == m.cols && (!eight || (m.cols % kGroup == 0 && m.scale_stride == m.cols / kGroup)));
}

int make_table(const ds_adamw_tensor *from, size_t n, ds_adamw &table) {
  std::vector<Tensor> tensors;
  std::vector<Range> written;
  std::vector<std::pair<uint32_t, uint32_t>> order;  // kind and place in `tensors`
  for (size_t k = 0; k < n; ++k) {
    const ds_adamw_tensor &f = from[k];
    bool copied = false;
    DS_TRY(check_tensor(f, copied));
    const int64_t rows = f.param.rows, cols = f.param.cols;
    if (rows == 0 || cols == 0) continue;
    const bool eight = f.m.dtype == DS_MX8;
    const ds_matrix *all[] = {&f.param, &f.grad, &f.m, &f.v, copied ? &f.copy : nullptr};
    bool row = true;
    for (const ds_matrix *m : all) {
      if (!m) continue;
      row = row && one_row(*m, m->dtype >= DS_MX8);
      if (m != &f.grad) add_range(written, m->base, rows, cols, m->row_stride, m->dtype >= DS_MX8 ? 1 : ds_itemsize(m->dtype));
      if (m->dtype >= DS_MX8) add_range(written, m->scale, rows, ds_groups(cols), m->scale_stride, 1);
    }
    Tensor t{};
    t.param = ds_rows(&f.param), t.grad = ds_rows(&f.grad), t.m = ds_rows(&f.m), t.v = ds_rows(&f.v), t.copy = ds_rows(copied ? &f.copy : nullptr);
    t.rows = row ? 1 : rows, t.cols = row ? rows * cols : cols;
    t.pieces = eight ? ds_groups(t.cols) * (kGroup / 8) : (t.cols + 7) / 8;
    t.number = (uint32_t)k, t.copy_dtype = copied ? f.copy.dtype : 0, t.decay = f.decay, t.rate = f.rate;
    order.emplace_back(f.param.dtype * 6 + f.grad.dtype * 2 + eight, (uint32_t)tensors.size());
    tensors.push_back(t);
  }
  if (written_twice(written)) return DS_EOVERLAP;
  std::stable_sort(order.begin(), order.end(), [](const auto &a, const auto &b) { return a.first < b.first; });
  std::vector<Chunk> chunks;
  for (size_t k = 0; k < order.size(); ++k) {
    const uint32_t kind = order[k].first, at = order[k].second;
    if (k == 0 || order[k - 1].first != kind) table.kinds.push_back({kind / 6, kind / 2 % 3, kind % 2, (int64_t)chunks.size(), 0});
    const int64_t all = tensors[at].rows * tensors[at].pieces;
    for (int64_t piece = 0; piece < all; piece += kPieces) chunks.push_back({piece, at, 0});
    table.kinds.back().end = (int64_t)chunks.size();
  }
  DS_HIP_TRY(hipGetDevice(&table.device));
  if (tensors.empty()) return DS_OK;
  const size_t first = tensors.size() * sizeof(Tensor), second = chunks.size() * sizeof(Chunk);
  const hipError_t e = hipMalloc(&table.memory, first + second);
  if (e == hipErrorOutOfMemory) {
    (void)hipGetLastError();
    return DS_ENOMEM;
  }
  DS_HIP_TRY(e);
  table.tensors = (const Tensor *)table.memory;
  table.chunks = (const Chunk *)((const uint8_t *)table.memory + first);
  DS_HIP_TRY(hipMemcpy(table.memory, tensors.data(), first, hipMemcpyHostToDevice));
  DS_HIP_TRY(hipMemcpy((uint8_t *)table.memory + first, chunks.data(), second, hipMemcpyHostToDevice));
  return DS_OK;
}

int on_its_device(const ds_adamw *table) {
  int device = -1;
  DS_HIP_TRY(hipGetDevice(&device));
  return device == table->device ? DS_OK : DS_ESTATE;
}

}  // namespace

extern "C" int ds_adamw_create(const ds_adamw_tensor *tensors, size_t n, ds_adamw **out) {
  if (!out || (n && !tensors)) return DS_EINVAL;
  if (n > 0xffffffffu) return DS_ERANGE;
  ds_adamw *table = new (std::nothrow) ds_adamw;
  if (!table) return DS_ENOMEM;
  int rc;
  try {
    rc = make_table(tensors, n, *table);
  } catch (const std::bad_alloc &) {
    rc = DS_ENOMEM;
  }
  if (rc != DS_OK) {
    if (table->memory) (void)hipFree(table->memory);
    delete table;
    return rc;
  }
  *out = table;
  return DS_OK;
}

extern "C" int ds_adamw_destroy(ds_adamw *table) {
  if (!table) return DS_EINVAL;
  int rc = DS_OK;
  if (table->memory) {
    const hipError_t e = hipFree(table->memory);
    if (e != hipSuccess) ds_set_hip_error(e), rc = DS_EHIP;
  }
  delete table;
  return rc;
}

extern "C" int ds_adamw_squares_workspace(const ds_adamw *table, uint64_t *bytes) {
  if (!table || !bytes) return DS_EINVAL;
  *bytes = (uint64_t)table->parts() * sizeof(double);
  return DS_OK;
}

extern "C" int ds_adamw_squares(const ds_adamw *table, double *squares, void *workspace, uint64_t workspace_bytes, void *stream) {
  if (!table || !squares || ds_misaligned(squares, 8)) return DS_EINVAL;
  const int64_t parts = table->parts();
  if (parts && (!workspace || ds_misaligned(workspace, 16))) return DS_EINVAL;
  if (workspace_bytes < (uint64_t)parts * sizeof(double)) return DS_ERANGE;
  DS_TRY(on_its_device(table));
  double *partial = (double *)workspace;
  for (const Kind &k : table->kinds) {
    const int64_t groups = square_groups(k);
    DS_TRY(ds_with_type(k.grad, [&](auto type) -> int {
      typedef decltype(type) G;
      hipLaunchKernelGGL(ds_adamw_squares_kernel<G>, dim3((uint32_t)groups), dim3(kThreads), 0, (hipStream_t)stream, table->tensors,
                         table->chunks + k.begin, k.end - k.begin, partial);
      DS_HIP_TRY(hipGetLastError());
      return DS_OK;
    }));
    partial += groups;
  }
  hipLaunchKernelGGL(ds_adamw_squares_sum_kernel, dim3(1), dim3(1024), 0, (hipStream_t)stream, (const double *)workspace, parts, squares);
  DS_HIP_TRY(hipGetLastError());
  return DS_OK;
}

extern "C" int ds_adamw_step(const ds_adamw *table, const ds_adamw_settings *settings, void *stream) {
  if (!table || !settings) return DS_EINVAL;
  const ds_adamw_settings &f = *settings;
  const auto share = [](double b) { return b >= 0.0 && b < 1.0; };
  const auto amount = [](double x) { return x >= 0.0 && x < (double)INFINITY; };
  if (!amount(f.rate) || !amount(f.eps) || !share(f.beta1) || !share(f.beta2) || !std::isfinite(f.grad_scale) || !(f.most_norm >= 0.0) || !f.step ||
      ds_misaligned(f.step, 8) || ds_misaligned(f.rate_now, 4) || ds_misaligned(f.squares, 8) || (f.most_norm > 0.0 && !f.squares))
    return DS_EINVAL;
  DS_TRY(on_its_device(table));
  const Settings s{f.rate, std::log(f.beta1), std::log(f.beta2), f.grad_scale, f.most_norm, f.step, f.rate_now, f.squares, (float)f.beta1,
                   (float)f.beta2, (float)(1.0 - f.beta1), (float)(1.0 - f.beta2), (float)f.eps, mix((uint32_t)f.seed ^ mix((uint32_t)(f.seed >> 32)))};
  for (const Kind &k : table->kinds) {
    const int64_t count = k.end - k.begin, grid = std::min(count, kMaxGrid);
    DS_TRY(ds_with_type(k.param, [&](auto type) -> int {
      typedef decltype(type) P;
      return ds_with_type(k.grad, [&](auto grad) -> int {
        typedef decltype(grad) G;
        const auto launch = [&](auto kernel) -> int {
          hipLaunchKernelGGL(kernel, dim3((uint32_t)grid), dim3(kThreads), 0, (hipStream_t)stream, table->tensors, table->chunks + k.begin, count, s);
          DS_HIP_TRY(hipGetLastError());
          return DS_OK;
        };
        return k.eight ? launch(ds_adamw_step_kernel<P, G, true>) : launch(ds_adamw_step_kernel<P, G, false>);
      });
    }));
  }
  return DS_OK;
}
