// Layer norm, forward and backward.
//
// Both are bound by HBM.  Forward: a work-group of 256 threads has a row, a thread pieces of eight columns 2048 apart; the
// mean is taken first and the squares of the differences from it then, so that a row whose mean is large beside its
// spread keeps its variance.  The row is read again for each of the three passes, out of the caches.  Backward: the same
// shape over several rows, each thread summing its columns' share of dgamma and dbeta over the work-group's rows; those
// sums are one line of `partial` each, and a second launch adds the lines in their order.

#include <type_traits>

#include "ds_ops.h"

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64, kStep = kThreads * 8;

// The sum over the work-group, in every thread.  `room`: one float per wavefront, free again after the next barrier.
__device__ inline float group_sum(float x, float *room) {
  x = wave_sum(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = x;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) s += room[w];
  return s;
}

struct NormForward {
  Rows x, y, saved;
  const void *gamma, *beta;
  float *mean, *rstd;
  int64_t rows, cols;
  float eps;
  uint32_t param_dtype;
};

template <typename T>
__global__ __launch_bounds__(kThreads) void ds_layernorm_forward_kernel(NormForward a) {
  __shared__ float room[kWaves];
  const auto count = [&](int64_t j) { return (int)(a.cols - j < 8 ? a.cols - j : 8); };
  for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x) {
    float sum = 0.f;
    for (int64_t j = threadIdx.x * 8; j < a.cols; j += kStep) {
      const Eight x = RowsOf<T>::get(a.x, i, j, count(j));
  #pragma unroll
      for (int k = 0; k < 8; ++k) sum += x.v[k];
    }
    const float mean = group_sum(sum, room) / (float)a.cols;
    float squares = 0.f;
    for (int64_t j = threadIdx.x * 8; j < a.cols; j += kStep) {
      const int n = count(j);
      const Eight x = RowsOf<T>::get(a.x, i, j, n);
  #pragma unroll
      for (int k = 0; k < 8; ++k) squares += k < n ? (x.v[k] - mean) * (x.v[k] - mean) : 0.f;
    }
    const float rstd = 1.f / sqrtf(group_sum(squares, room) / (float)a.cols + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[i] = mean;
      if (a.rstd) a.rstd[i] = rstd;
    }
    for (int64_t first = 0; first < a.cols; first += kStep) {
      const int64_t j = first + threadIdx.x * 8;
      const int n = j < a.cols ? count(j) : 0;
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
  float *partial;  // [2 * parts][cols]: dgamma's lines, then dbeta's; or NULL
  int64_t rows, cols;
  uint32_t param_dtype;
};

// A row's sums and dx; the work-groups stride over the rows.
template <typename T, typename X>
__global__ __launch_bounds__(kThreads) void ds_layernorm_backward_kernel(NormBackward a) {
  __shared__ float room[kWaves];
  const auto count = [&](int64_t j) { return (int)(a.cols - j < 8 ? a.cols - j : 8); };
  for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x) {
    const float mean = a.mean[i], rstd = a.rstd[i];
    float flat = 0.f, along = 0.f;
    for (int64_t j = threadIdx.x * 8; j < a.cols; j += kStep) {
      const int n = count(j);
      const Eight d = RowsOf<T>::get(a.dy, i, j, n), x = RowsOf<X>::get(a.x, i, j, n), g = get_up_to8_any(a.gamma, a.param_dtype, j, n, 1.f);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float w = d.v[k] * g.v[k];
        flat += w;
        along += k < n ? w * ((x.v[k] - mean) * rstd) : 0.f;
      }
    }
    flat = group_sum(flat, room) / (float)a.cols;
    along = group_sum(along, room) / (float)a.cols;
    for (int64_t j = threadIdx.x * 8; j < a.cols; j += kStep) {
      const int n = count(j);
      const Eight d = RowsOf<T>::get(a.dy, i, j, n), x = RowsOf<X>::get(a.x, i, j, n), g = get_up_to8_any(a.gamma, a.param_dtype, j, n, 1.f);
      Eight r = {};
      if (a.residual.base) r = RowsOf<T>::get(a.residual, i, j, n);
#pragma unroll
      for (int k = 0; k < 8; ++k) r.v[k] += rstd * (d.v[k] * g.v[k] - flat - (x.v[k] - mean) * rstd * along);
      put_up_to8<T>(a.dx.base, i * a.dx.stride + j, n, r);
    }
  }
}

// dgamma's and dbeta's lines: a work-group has 512 columns and every (4 * parts)-th row for each of its wavefronts.
template <typename T, typename X>
__global__ __launch_bounds__(kThreads) void ds_layernorm_param_kernel(NormBackward a) {
  __shared__ float sums[2][kWaves][64][8 + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t j = ((int64_t)blockIdx.x * 64 + lane) * 8, left = a.cols - j;
  const int n = (int)(left < 0 ? 0 : left < 8 ? left : 8);
  Eight dg = {}, db = {};
  for (int64_t i = (int64_t)blockIdx.y * kWaves + wave; i < a.rows; i += (int64_t)gridDim.y * kWaves) {
    const float mean = a.mean[i], rstd = a.rstd[i];
    const Eight d = RowsOf<T>::get(a.dy, i, j, n), x = RowsOf<X>::get(a.x, i, j, n);
#pragma unroll
    for (int k = 0; k < 8; ++k) dg.v[k] += d.v[k] * ((x.v[k] - mean) * rstd), db.v[k] += d.v[k];
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) sums[0][wave][lane][k] = dg.v[k], sums[1][wave][lane][k] = db.v[k];
  __syncthreads();
  for (int c = threadIdx.x; c < 1024; c += kThreads) {
    const int which = c / 512, at = c % 512;
    const int64_t col = (int64_t)blockIdx.x * 512 + at;
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s += sums[which][w][at / 8][at % 8];
    if (col < a.cols) a.partial[((int64_t)which * gridDim.y + blockIdx.y) * a.cols + col] = s;
  }
}

int64_t norm_parts(int64_t rows, int64_t cols) {
  const int64_t across = cols > 512 ? (cols + 511) / 512 : 1, by_rows = (rows + kWaves - 1) / kWaves, by_grid = (1024 + across - 1) / across;
  const int64_t parts = by_rows < by_grid ? by_rows : by_grid;
  return parts < 1 ? 1 : parts;
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
    hipLaunchKernelGGL(ds_layernorm_forward_kernel<T>, dim3((uint32_t)(a.rows < kMaxGrid ? a.rows : kMaxGrid)), dim3(kThreads), 0, (hipStream_t)stream, a);
    DS_HIP_TRY(hipGetLastError());
    return DS_OK;
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
  const NormBackward a{ds_rows(dy), ds_rows(x), ds_rows(residual), ds_rows(dx), mean, rstd, gamma, (float *)workspace, rows, cols, param_dtype};
  if (rows > 0) {
    const int rc = ds_with_type(dy->dtype, [&](auto type) -> int {
      typedef decltype(type) T;
      const dim3 grid((uint32_t)((cols + 511) / 512), (uint32_t)parts), row_grid((uint32_t)(rows < 4096 ? rows : 4096));
      const auto launch = [&](auto params, auto norm) {
        // the parameters' sums first: dx may be dy
        if (sums) hipLaunchKernelGGL(params, grid, dim3(kThreads), 0, st, a);
        hipLaunchKernelGGL(norm, row_grid, dim3(kThreads), 0, st, a);
      };
      if (x->dtype == DS_MX8) launch(ds_layernorm_param_kernel<T, Mx8>, ds_layernorm_backward_kernel<T, Mx8>);
      else launch(ds_layernorm_param_kernel<T, T>, ds_layernorm_backward_kernel<T, T>);
      DS_HIP_TRY(hipGetLastError());
      return DS_OK;
    });
    DS_TRY(rc);
  }
  const int64_t lines = rows > 0 ? parts : 0;
  if (dgamma) DS_TRY(ds_launch_sum_parts((const float *)workspace, lines, cols, dgamma, st));
  if (dbeta) DS_TRY(ds_launch_sum_parts((const float *)workspace + lines * cols, lines, cols, dbeta, st));
  return DS_OK;
}
