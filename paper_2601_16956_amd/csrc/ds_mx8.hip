// Checkpoints of activations in 8 bits: written, read back, and the backward pass of an activation that reads one.
//
// All three are bound by HBM: a few operations for each value that is read or written once.  A lane holds eight
// neighbouring columns, which is one 16-byte access of a 16-bit type and 8 bytes of codes, and four lanes a group of 32
// that shares a scale: its largest magnitude is two moves between lanes of a quad, and the scale is one byte that the
// first of the four writes.  The scale is a power of two, so that x / step is exact before it is rounded to a whole number
// and the value that is read back has at most 7 significant bits, which every type holds.
//
// 8192 x 8192 bfloat16: written in 44 us (203 MB, 4.6 TB/s), read back in 32 us (6.3 TB/s).  The activation's backward pass, silu on 16384
// x 3584, 60 us (295 MB, 4.9 TB/s), by GELU's erf form 64: of these, three are of the last 3 of 2051 work-groups, which wait for the 2048 that
// run at once.

#include <type_traits>

#include "ds_ops.h"

namespace {

constexpr int kThreads = 256;

// Work items are pieces of eight columns; a row has a multiple of four of them, so that a group's are four neighbouring lanes.
// (A division in 64 bits takes as long as the rest.  Index: uint32_t where it holds their number; `shift` is the binary logarithm of
// `pieces`, or -1 where that is none.)
template <typename T, typename Index>
__global__ __launch_bounds__(kThreads) void ds_mx8_save_kernel(Rows x, Rows saved, int64_t rows, int64_t cols, uint32_t pieces, int shift) {
  for (int64_t first = (int64_t)blockIdx.x * kThreads; first < rows * pieces; first += (int64_t)gridDim.x * kThreads) {
    const Index item = (Index)(first + threadIdx.x), row = shift >= 0 ? item >> shift : item / (Index)pieces;
    const int64_t i = row, j = (int64_t)(item - row * (Index)pieces) * 8, left = i < rows ? cols - j : 0;
    const int n = (int)(left < 0 ? 0 : left < 8 ? left : 8);
    mx8_put(saved, i, j, n, RowsOf<T>::get(x, i, j, n));
  }
}

template <typename T, typename Index>
__global__ __launch_bounds__(kThreads) void ds_mx8_load_kernel(Rows saved, Rows x, int64_t rows, int64_t cols, uint32_t pieces, int shift) {
  for (int64_t first = (int64_t)blockIdx.x * kThreads; first < rows * pieces; first += (int64_t)gridDim.x * kThreads) {
    const Index item = (Index)(first + threadIdx.x), row = shift >= 0 ? item >> shift : item / (Index)pieces;
    const int64_t i = row, j = (int64_t)(item - row * (Index)pieces) * 8, left = i < rows ? cols - j : 0;
    const int n = (int)(left < 0 ? 0 : left < 8 ? left : 8);
    put_up_to8<T>(x.base, i * x.stride + j, n, RowsOf<Mx8>::get(saved, i, j, n));
  }
}

int check_pair(const ds_matrix *x, const ds_matrix *saved) {
  DS_TRY(ds_check_matrix(x, true));
  DS_TRY(ds_check_matrix(saved, true));
  return x->dtype == DS_MX8 || saved->dtype != DS_MX8 || !ds_same_extents(x, saved) ? DS_EINVAL : DS_OK;
}

template <bool SAVE>
int launch_mx8(const ds_matrix *x, const ds_matrix *saved, hipStream_t stream) {
  DS_TRY(check_pair(x, saved));
  if (x->rows == 0 || x->cols == 0) return DS_OK;
  const int64_t pieces = ds_groups(x->cols) * (kGroup / 8), all = (x->rows * pieces + kThreads - 1) / kThreads;
  const int64_t grid = all < kMaxGrid ? all : kMaxGrid;
  const int shift = (pieces & (pieces - 1)) == 0 ? __builtin_ctzll(pieces) : -1;
  const bool narrow = all <= (int64_t)0xffffffff / kThreads;
  return ds_with_type(x->dtype, [&](auto type) -> int {
    typedef decltype(type) T;
    const auto launch = [&](auto kernel, const ds_matrix *from, const ds_matrix *to) -> int {
      hipLaunchKernelGGL(kernel, dim3((uint32_t)grid), dim3(kThreads), 0, stream, ds_rows(from), ds_rows(to), x->rows, x->cols, (uint32_t)pieces, shift);
      DS_HIP_TRY(hipGetLastError());
      return DS_OK;
    };
    if (SAVE) return narrow ? launch(ds_mx8_save_kernel<T, uint32_t>, x, saved) : launch(ds_mx8_save_kernel<T, uint64_t>, x, saved);
    return narrow ? launch(ds_mx8_load_kernel<T, uint32_t>, saved, x) : launch(ds_mx8_load_kernel<T, uint64_t>, saved, x);
  });
}

// A work-group takes 64 pieces of eight columns and every (4 * parts)-th row of them for each of its four wavefronts, which ask for the
// next row before they compute on this one; the sums over its rows are one line of `partial`.
template <typename T, typename Z, uint32_t ACT>
__global__ __launch_bounds__(kThreads) void ds_activation_backward_kernel(Rows dy, Rows z, Rows dz, int64_t rows, int64_t cols,
                                                                          float *partial) {
  __shared__ float sums[4][64][8 + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t j = ((int64_t)blockIdx.x * 64 + lane) * 8, left = cols - j, stride = (int64_t)gridDim.y * 4;
  const int n = (int)(left < 0 ? 0 : left < 8 ? left : 8);
  Eight sum = {};
  int64_t i = (int64_t)blockIdx.y * 4 + wave;
  auto next_d = RowsOf<T>::ask(dy, i, j, i < rows ? n : 0);
  auto next_at = RowsOf<Z>::ask(z, i, j, i < rows ? n : 0);
  for (; i < rows; i += stride) {
    const Eight d = RowsOf<T>::value(next_d, n), at = RowsOf<Z>::value(next_at, n);
    const int more = i + stride < rows ? n : 0;
    next_d = RowsOf<T>::ask(dy, i + stride, j, more), next_at = RowsOf<Z>::ask(z, i + stride, j, more);
    Eight r;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      r.v[k] = d.v[k] * activation_slope<ACT, sizeof(T) == 4>(at.v[k]);
      sum.v[k] += k < n ? r.v[k] : 0.f;
    }
    put_up_to8<T>(dz.base, i * dz.stride + j, n, r);
  }
  if (!partial) return;
#pragma unroll
  for (int k = 0; k < 8; ++k) sums[wave][lane][k] = sum.v[k];
  __syncthreads();
  for (int c = threadIdx.x; c < 512; c += kThreads) {
    const int64_t col = (int64_t)blockIdx.x * 512 + c;
    if (col < cols)
      partial[blockIdx.y * cols + col] = sums[0][c / 8][c % 8] + sums[1][c / 8][c % 8] + sums[2][c / 8][c % 8] + sums[3][c / 8][c % 8];
  }
}

// The lines of `partial` added: a work-group has 16 columns (and further ones where a launch has no place for as many work-groups), and each
// of its 16 rows of threads every 16th line; then those 16 sums in their order.  blockIdx.y: the first or the second set of lines.
__global__ __launch_bounds__(kThreads) void ds_sum_parts_kernel(const float *partial, int64_t parts, int64_t cols, float *out0, float *out1) {
  __shared__ float sums[16][16 + 1];
  const int across = threadIdx.x % 16, row = threadIdx.x / 16;
  float *out = blockIdx.y ? out1 : out0;
  if (!out) return;
  for (int64_t first = (int64_t)blockIdx.x * 16; first < cols; first += (int64_t)gridDim.x * 16) {
    const int64_t j = first + across;
    const float *from = partial + blockIdx.y * parts * cols + j;
    float sum[4] = {};
    if (j < cols) {
      int64_t p = row;
      for (; p + 48 < parts; p += 64)
#pragma unroll
        for (int u = 0; u < 4; ++u) sum[u] += from[(p + 16 * u) * cols];
      for (; p < parts; p += 16) sum[0] += from[p * cols];
    }
    sums[row][across] = sum[0] + sum[1] + (sum[2] + sum[3]);
    __syncthreads();
    if (row == 0 && j < cols) {
      float s = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) s += sums[r][across];
      out[j] = s;
    }
    __syncthreads();
  }
}

// Few rows: a work-group has 64 columns, eight lanes a row of them and 128 rows at a time, and sums the bias's gradient itself: one launch.
// So / by the kernel above and the sum of its lines, us of the GPU, silu on bfloat16 from 8 bits: 1 x 1024 3.8 / 5.1, 128 x 1024 4.4 / 5.6, 256 x
// 1024 5.3 / 5.5, 333 x 1024 6.3 / 6.1, 384 x 1024 6.8 / 6.3 and 512 x 1024 7.2 / 5.7; 384 x 256 6.1 / 6.1, 384 x 4096 7.3 / 8.3, 1 x 16384
// 4.1 / 5.5, 384 x 16384 10.9 / 14.5.  A caller who does not wait in between has a launch less: 333 x 1024 10.8 / 14.2.
constexpr int64_t kFewRows = 384, kFewCols = 16384;
template <typename T, typename Z, uint32_t ACT>
__global__ __launch_bounds__(1024) void ds_activation_backward_few_kernel(Rows dy, Rows z, Rows dz, int rows, int64_t cols, float *dbias) {
  __shared__ float sums[128][64 + 1];
  const int across = threadIdx.x % 8, row = threadIdx.x / 8;
  const int64_t j = (int64_t)blockIdx.x * 64 + across * 8, left = cols - j;
  const int n = (int)(left < 0 ? 0 : left < 8 ? left : 8);
  constexpr int kTimes = (int)kFewRows / 128;
  typename RowsOf<T>::Bits d[kTimes];
  typename RowsOf<Z>::Bits at[kTimes];
#pragma unroll
  for (int u = 0; u < kTimes; ++u) {
    const int i = u * 128 + row;
    d[u] = RowsOf<T>::ask(dy, i, j, i < rows ? n : 0), at[u] = RowsOf<Z>::ask(z, i, j, i < rows ? n : 0);
  }
  Eight sum = {};
#pragma unroll
  for (int u = 0; u < kTimes; ++u) {
    const int i = u * 128 + row;
    if (i >= rows) break;
    const Eight g = RowsOf<T>::value(d[u], n), x = RowsOf<Z>::value(at[u], n);
    Eight r;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      r.v[k] = g.v[k] * activation_slope<ACT, sizeof(T) == 4>(x.v[k]);
      sum.v[k] += k < n ? r.v[k] : 0.f;
    }
    put_up_to8<T>(dz.base, i * dz.stride + j, n, r);
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) sums[row][across * 8 + k] = sum.v[k];
  // 128 sums of a column, 16 lanes eight of them each, then those 16 in their order
  __syncthreads();
  const int column = threadIdx.x / 16, part = threadIdx.x % 16;
  float s = 0.f;
#pragma unroll
  for (int r = 0; r < 8; ++r) s += sums[part * 8 + r][column];
  __syncthreads();
  sums[part][column] = s;
  __syncthreads();
  if (threadIdx.x < 64 && (int64_t)blockIdx.x * 64 + threadIdx.x < cols) {
    float total = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) total += sums[r][threadIdx.x];
    dbias[(int64_t)blockIdx.x * 64 + threadIdx.x] = total;
  }
}

constexpr int64_t kActGroups = 2048;  // work-groups of a launch, about
int64_t act_parts(int64_t rows, int64_t cols) {
  const int64_t across = cols > 512 ? (cols + 511) / 512 : 1, by_rows = (rows + 3) / 4, by_grid = (kActGroups + across - 1) / across;
  const int64_t parts = by_rows < by_grid ? by_rows : by_grid;
  return parts < 1 ? 1 : parts > 65535 ? 65535 : parts;
}

}  // namespace

int ds_launch_sum_parts(const float *partial, int64_t parts, int64_t cols, float *out0, float *out1, hipStream_t stream) {
  const int64_t groups = (cols + 15) / 16;
  hipLaunchKernelGGL(ds_sum_parts_kernel, dim3((uint32_t)(groups < kMaxGrid ? groups : kMaxGrid), out1 ? 2 : 1), dim3(kThreads), 0, stream, partial,
                     parts, cols, out0, out1);
  DS_HIP_TRY(hipGetLastError());
  return DS_OK;
}

extern "C" int ds_mx8_save(const ds_matrix *x, const ds_matrix *saved, void *stream) {
  return launch_mx8<true>(x, saved, (hipStream_t)stream);
}

extern "C" int ds_mx8_load(const ds_matrix *saved, const ds_matrix *x, void *stream) {
  return launch_mx8<false>(x, saved, (hipStream_t)stream);
}

extern "C" int ds_activation_backward_workspace(int64_t rows, int64_t cols, uint64_t *bytes) {
  if (!bytes || rows < 0 || cols < 0) return DS_EINVAL;
  if (rows > kMaxExtent || cols > kMaxExtent) return DS_ERANGE;
  *bytes = (uint64_t)(act_parts(rows, cols) * cols * 4);
  return DS_OK;
}

extern "C" int ds_activation_backward(const ds_matrix *dy, const ds_matrix *z, uint32_t act, const ds_matrix *dz, float *dbias,
                                      void *workspace, uint64_t workspace_bytes, void *stream) {
  DS_TRY(ds_check_matrix(dy, true));
  DS_TRY(ds_check_matrix(z, true));
  DS_TRY(ds_check_matrix(dz, true));
  if (dy->dtype == DS_MX8 || dz->dtype != dy->dtype || (z->dtype != DS_MX8 && z->dtype != dy->dtype) || act > DS_ACT_SILU ||
      !ds_same_extents(dy, z) || !ds_same_extents(dy, dz) || ds_misaligned(dbias, 4))
    return DS_EINVAL;
  const int64_t rows = dy->rows, cols = dy->cols, parts = act_parts(rows, cols);
  if (cols == 0 || (rows == 0 && !dbias)) return DS_OK;
  if (dbias) {
    if (!workspace || ds_misaligned(workspace, 16)) return DS_EINVAL;
    if (workspace_bytes < (uint64_t)(parts * cols * 4)) return DS_ERANGE;
  }
  hipStream_t st = (hipStream_t)stream;
  const bool few = dbias && rows > 0 && rows <= kFewRows && cols <= kFewCols;
  if (rows > 0) {
    const dim3 grid((uint32_t)((cols + 511) / 512), (uint32_t)parts);
    const int rc = ds_with_type(dy->dtype, [&](auto type) -> int {
      typedef decltype(type) T;
      return ds_with_act(act, [&](auto a) -> int {
        constexpr uint32_t A = decltype(a)::value;
        if (few) {
          const auto launch = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((uint32_t)((cols + 63) / 64)), dim3(1024), 0, st, ds_rows(dy), ds_rows(z), ds_rows(dz), (int)rows, cols, dbias);
          };
          if (z->dtype == DS_MX8) launch(ds_activation_backward_few_kernel<T, Mx8, A>);
          else launch(ds_activation_backward_few_kernel<T, T, A>);
        } else if (z->dtype == DS_MX8)
          hipLaunchKernelGGL((ds_activation_backward_kernel<T, Mx8, A>), grid, dim3(kThreads), 0, st, ds_rows(dy), ds_rows(z),
                             ds_rows(dz), rows, cols, dbias ? (float *)workspace : nullptr);
        else
          hipLaunchKernelGGL((ds_activation_backward_kernel<T, T, A>), grid, dim3(kThreads), 0, st, ds_rows(dy), ds_rows(z),
                             ds_rows(dz), rows, cols, dbias ? (float *)workspace : nullptr);
        DS_HIP_TRY(hipGetLastError());
        return DS_OK;
      });
    });
    DS_TRY(rc);
  }
  return dbias && !few ? ds_launch_sum_parts((const float *)workspace, rows > 0 ? parts : 0, cols, dbias, nullptr, st) : DS_OK;
}
