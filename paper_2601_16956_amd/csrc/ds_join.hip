// A block's output joined to the residual stream, with a norm behind the block, a gate, the residual's scale and a norm in front of
// the next block; forward and backward.
//
// Both are bound by HBM: forward reads u and x and writes out and y, backward reads dout, dy, u and out and writes du and dx,
// each once.  As in layer norm, a row belongs to one to sixteen wavefronts, whose threads hold it in registers in pieces of
// eight neighbouring columns; a work-group walks over several rows.  Backward, a thread also sums its columns' share of
// the two sums over rows that all three parameters' gradients come from,
//   a_j = sum dy * h  and  b_j = sum d * k:  dbefore = a,  dgate = scale * after_gamma * b,  dafter = scale * gate * b;
// they are a line for each work-group, and a second launch adds the lines in their order.
// Rows too long for the registers are read again for every pass.

#include <type_traits>

#include "ds_ops.h"

namespace {

__device__ inline int columns_left(int64_t cols, int64_t j) {
  const int64_t left = cols - j;
  return (int)(left < 0 ? 0 : left < 8 ? left : 8);
}

// The sum of `x` over the `WAVES` wavefronts of a row, in every thread.  `room`: one float per wavefront, another one in every turn: it is
// written again only behind the barrier of a sum in between.
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

struct Vectors {
  const void *after_gamma, *gate, *before_gamma;
  uint32_t dtype;
  float keep, scale, eps;
};
// scale * gate * after_gamma
__device__ inline Eight weight_of(const Vectors &v, int64_t j, int n) {
  const Eight gate = get_up_to8_any(v.gate, v.dtype, j, n, 1.f), gamma = get_up_to8_any(v.after_gamma, v.dtype, j, n, 1.f);
  Eight w;
#pragma unroll
  for (int k = 0; k < 8; ++k) w.v[k] = v.scale * gate.v[k] * gamma.v[k];
  return w;
}

// What eight elements of out are when they are read back.
template <typename T>
__device__ inline void as_stored(Eight &e) {
  typename RowsOf<T>::Bits b;
  Elem<T>::put8(&b, 0, e);
  e = RowsOf<T>::value(b, 8);
}

struct JoinForward {
  Rows u, x, out, y;
  Vectors v;
  float *rstd_after, *rstd_before;
  int64_t rows, cols;
  bool after, before;
};

// WAVES wavefronts have a row, each thread HAS pieces of eight columns, 512 * WAVES apart; a work-group of WIDE wavefronts has
// WIDE / WAVES rows at a time.  AHEAD: it asks for the next row before it computes on this one, where the registers hold both.
template <typename T, int WAVES, int WIDE, int HAS, bool AHEAD = true>
__global__ __launch_bounds__(WIDE * 64) void ds_join_forward_kernel(JoinForward a) {
  __shared__ float room[2][2][WIDE];
  constexpr int kRows = WIDE / WAVES, kApart = WAVES * 512;
  const int at = threadIdx.x % (WAVES * 64) * 8, which = threadIdx.x / (WAVES * 64);
  const bool joins = a.u.base != nullptr;
  const float each = 1.f / (float)a.cols;
  const int64_t stride = (int64_t)gridDim.x * kRows;
  int64_t i = (int64_t)blockIdx.x * kRows + which;
  int n[HAS];
  typename RowsOf<T>::Bits next_x[HAS], next_u[HAS] = {};
  const auto ask = [&](int64_t i) {
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
      const int has = i < a.rows ? n[p] : 0;
      next_x[p] = RowsOf<T>::ask(a.x, i, at + p * kApart, has);
      if (joins) next_u[p] = RowsOf<T>::ask(a.u, i, at + p * kApart, has);
    }
  };
#pragma unroll
  for (int p = 0; p < HAS; ++p) n[p] = columns_left(a.cols, at + p * kApart);
  if (AHEAD) ask(i);
  Eight w[HAS], g[HAS];
#pragma unroll
  for (int p = 0; p < HAS; ++p) {
    w[p] = weight_of(a.v, at + p * kApart, n[p]);
    g[p] = get_up_to8_any(a.v.before_gamma, a.v.dtype, at + p * kApart, n[p], 1.f);
  }
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.rows; first += stride, i += stride, turn ^= 1) {
    Eight x[HAS], u[HAS];
    float squares = 0.f;
    if (!AHEAD) ask(i);
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
      x[p] = RowsOf<T>::value(next_x[p], n[p]), u[p] = RowsOf<T>::value(next_u[p], n[p]);
#pragma unroll
      for (int k = 0; k < 8; ++k) squares += u[p].v[k] * u[p].v[k];
    }
    if (AHEAD) ask(i + stride);
    const bool row = i < a.rows;
    float after = 1.f;
    if (a.after) {
      after = 1.f / sqrtf(row_sum<WAVES>(squares, room[turn][0]) * each + a.v.eps);
      if (row && at == 0 && a.rstd_after) a.rstd_after[i] = after;
    }
    squares = 0.f;
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
      if (joins) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[p].v[k] = a.v.keep * x[p].v[k] + u[p].v[k] * after * w[p].v[k];
        as_stored<T>(x[p]);
        if (row && a.out.base) put_up_to8<T>(a.out.base, i * a.out.stride + at + p * kApart, n[p], x[p]);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) squares += k < n[p] ? x[p].v[k] * x[p].v[k] : 0.f;
    }
    if (!a.before) continue;
    const float before = 1.f / sqrtf(row_sum<WAVES>(squares, room[turn][1]) * each + a.v.eps);
    if (!row) continue;
    if (at == 0 && a.rstd_before) a.rstd_before[i] = before;
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[p].v[k] = x[p].v[k] * before * g[p].v[k];
      put_up_to8<T>(a.y.base, i * a.y.stride + at + p * kApart, n[p], x[p]);
    }
  }
}

// Rows of any length.  (A thread has the same columns in every pass, so that out may be x, and y may be u.)
template <typename T>
__global__ __launch_bounds__(1024) void ds_join_forward_long_kernel(JoinForward a) {
  __shared__ float room[2][2][16];
  constexpr int kApart = 1024 * 8;
  const bool joins = a.u.base != nullptr;
  const float each = 1.f / (float)a.cols;
  int turn = 0;
  for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x, turn ^= 1) {
    float after = 1.f, squares = 0.f;
    if (a.after) {
      for (int64_t j = threadIdx.x * 8; j < a.cols; j += kApart) {
        const Eight u = RowsOf<T>::get(a.u, i, j, columns_left(a.cols, j));
#pragma unroll
        for (int k = 0; k < 8; ++k) squares += u.v[k] * u.v[k];
      }
      after = 1.f / sqrtf(row_sum<16>(squares, room[turn][0]) * each + a.v.eps);
      if (threadIdx.x == 0 && a.rstd_after) a.rstd_after[i] = after;
    }
    squares = 0.f;
    for (int64_t j = threadIdx.x * 8; j < a.cols; j += kApart) {
      const int n = columns_left(a.cols, j);
      Eight x = RowsOf<T>::get(a.x, i, j, n);
      if (joins) {
        const Eight u = RowsOf<T>::get(a.u, i, j, n), w = weight_of(a.v, j, n);
#pragma unroll
        for (int k = 0; k < 8; ++k) x.v[k] = a.v.keep * x.v[k] + u.v[k] * after * w.v[k];
        as_stored<T>(x);
        put_up_to8<T>(a.out.base, i * a.out.stride + j, n, x);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) squares += k < n ? x.v[k] * x.v[k] : 0.f;
    }
    if (!a.before) continue;
    const float before = 1.f / sqrtf(row_sum<16>(squares, room[turn][1]) * each + a.v.eps);
    if (threadIdx.x == 0 && a.rstd_before) a.rstd_before[i] = before;
    for (int64_t j = threadIdx.x * 8; j < a.cols; j += kApart) {
      const int n = columns_left(a.cols, j);
      Eight x = RowsOf<T>::get(joins ? a.out : a.x, i, j, n);
      const Eight g = get_up_to8_any(a.v.before_gamma, a.v.dtype, j, n, 1.f);
#pragma unroll
      for (int k = 0; k < 8; ++k) x.v[k] = x.v[k] * before * g.v[k];
      put_up_to8<T>(a.y.base, i * a.y.stride + j, n, x);
    }
  }
}

struct JoinBackward {
  Rows dout, dy, u, out, du, dx;
  Vectors v;
  const float *rstd_after, *rstd_before;
  float *partial;  // [2][parts][cols]: lines of a, then of b; or NULL
  int64_t rows, cols;
  bool after, before;
};

// The shapes are the forward kernel's.
template <typename T, int WAVES, int WIDE, int HAS>
__global__ __launch_bounds__(WIDE * 64) void ds_join_backward_kernel(JoinBackward a) {
  constexpr int kRows = WIDE / WAVES, kApart = WAVES * 512;
  __shared__ float room[2][2][WIDE];
  __shared__ float lines[kRows > 1 ? kRows : 1][kRows > 1 ? HAS * kApart : 1];
  const int at = threadIdx.x % (WAVES * 64) * 8, which = threadIdx.x / (WAVES * 64);
  const bool joins = a.u.base != nullptr;
  const float each = 1.f / (float)a.cols;
  const int64_t stride = (int64_t)gridDim.x * kRows;
  Eight g[HAS], w[HAS], da[HAS] = {}, db[HAS] = {};
  int n[HAS];
#pragma unroll
  for (int p = 0; p < HAS; ++p) {
    n[p] = columns_left(a.cols, at + p * kApart);
    g[p] = get_up_to8_any(a.v.before_gamma, a.v.dtype, at + p * kApart, n[p], 1.f);
    w[p] = weight_of(a.v, at + p * kApart, n[p]);
  }
  int64_t i = (int64_t)blockIdx.x * kRows + which;
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.rows; first += stride, i += stride, turn ^= 1) {
    const bool row = i < a.rows;
    typename RowsOf<T>::Bits bits_d[HAS] = {}, bits_u[HAS] = {}, bits_y[HAS] = {}, bits_o[HAS] = {};
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
      const int64_t j = at + p * kApart;
      const int has = row ? n[p] : 0;
      if (a.dout.base) bits_d[p] = RowsOf<T>::ask(a.dout, i, j, has);
      if (a.before) bits_y[p] = RowsOf<T>::ask(a.dy, i, j, has), bits_o[p] = RowsOf<T>::ask(a.out, i, j, has);
      if (joins) bits_u[p] = RowsOf<T>::ask(a.u, i, j, has);
    }
    const float before = a.before && row ? a.rstd_before[i] : 0.f, after = a.after && row ? a.rstd_after[i] : 1.f;
    Eight d[HAS];
    float along = 0.f;
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
      d[p] = RowsOf<T>::value(bits_d[p], 8);
      if (!a.before) continue;
      const Eight dy = RowsOf<T>::value(bits_y[p], 8), o = RowsOf<T>::value(bits_o[p], 8);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float h = o.v[k] * before;
        da[p].v[k] += dy.v[k] * h;
        along += dy.v[k] * g[p].v[k] * h;
      }
    }
    if (a.before) {
      along = row_sum<WAVES>(along, room[turn][0]) * each;
#pragma unroll
      for (int p = 0; p < HAS; ++p) {
        const Eight dy = RowsOf<T>::value(bits_y[p], 8), o = RowsOf<T>::value(bits_o[p], 8);
#pragma unroll
        for (int k = 0; k < 8; ++k) d[p].v[k] += before * (dy.v[k] * g[p].v[k] - o.v[k] * before * along);
      }
    }
    if (row && a.dx.base) {
#pragma unroll
      for (int p = 0; p < HAS; ++p) {
        Eight dx;
#pragma unroll
        for (int k = 0; k < 8; ++k) dx.v[k] = joins ? a.v.keep * d[p].v[k] : d[p].v[k];
        put_up_to8<T>(a.dx.base, i * a.dx.stride + at + p * kApart, n[p], dx);
      }
    }
    if (!joins) continue;
    along = 0.f;
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
      const Eight u = RowsOf<T>::value(bits_u[p], 8);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float b = d[p].v[k] * (u.v[k] * after);
        db[p].v[k] += b;
        along += b * w[p].v[k];
      }
    }
    along = a.after ? row_sum<WAVES>(along, room[turn][1]) * each : 0.f;
    if (!row || !a.du.base) continue;
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
      Eight du = RowsOf<T>::value(bits_u[p], 8);
#pragma unroll
      for (int k = 0; k < 8; ++k) du.v[k] = after * (d[p].v[k] * w[p].v[k] - du.v[k] * after * along);
      put_up_to8<T>(a.du.base, i * a.du.stride + at + p * kApart, n[p], du);
    }
  }
  if (!a.partial) return;
  const int64_t parts = gridDim.x;
  if (kRows == 1) {
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
      const int64_t j = at + p * kApart;
      put_up_to8<float>(a.partial, blockIdx.x * a.cols + j, n[p], da[p]);
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
      for (int k = 0; k < 8; ++k) lines[which][at + p * kApart + k] = s ? db[p].v[k] : da[p].v[k];
    __syncthreads();
    for (int j = threadIdx.x; j < a.cols; j += WIDE * 64) {
      float sum = 0.f;
#pragma unroll
      for (int r = 0; r < kRows; ++r) sum += lines[r][j];
      a.partial[(s * parts + blockIdx.x) * a.cols + j] = sum;
    }
  }
}

// Rows of any length: the gradient of the stream behind the joint, and the terms of both sums.
struct LongRow {
  float before, after, along;  // `along`: of the norm in front of the next block
};
template <typename T>
__device__ inline Eight stream_gradient(const JoinBackward &a, const LongRow &r, int64_t i, int64_t j, int n, Eight &term) {
  Eight d = {};
  term = Eight{};
  if (a.dout.base) d = RowsOf<T>::get(a.dout, i, j, n);
  if (a.before) {
    const Eight dy = RowsOf<T>::get(a.dy, i, j, n), o = RowsOf<T>::get(a.out, i, j, n);
    const Eight g = get_up_to8_any(a.v.before_gamma, a.v.dtype, j, n, 1.f);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float h = o.v[k] * r.before;
      term.v[k] = dy.v[k] * h;
      d.v[k] += r.before * (dy.v[k] * g.v[k] - h * r.along);
    }
  }
  return d;
}

// A row's sums, du and dx.  `alongs`: [rows] the sums of the norm in front of the next block, for the parameters' kernel.
template <typename T>
__global__ __launch_bounds__(1024) void ds_join_backward_long_kernel(JoinBackward a, float *alongs, bool sums_only) {
  __shared__ float room[2][2][16];
  constexpr int kApart = 1024 * 8;
  const bool joins = a.u.base != nullptr;
  const float each = 1.f / (float)a.cols;
  int turn = 0;
  for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x, turn ^= 1) {
    LongRow r = {a.before ? a.rstd_before[i] : 0.f, a.after ? a.rstd_after[i] : 1.f, 0.f};
    if (sums_only || !alongs) {
      float along = 0.f;
      if (a.before) {
        for (int64_t j = threadIdx.x * 8; j < a.cols; j += kApart) {
          const int n = columns_left(a.cols, j);
          const Eight dy = RowsOf<T>::get(a.dy, i, j, n), o = RowsOf<T>::get(a.out, i, j, n);
          const Eight g = get_up_to8_any(a.v.before_gamma, a.v.dtype, j, n, 1.f);
#pragma unroll
          for (int k = 0; k < 8; ++k) along += dy.v[k] * g.v[k] * (o.v[k] * r.before);
        }
        r.along = row_sum<16>(along, room[turn][0]) * each;
      }
    } else {
      r.along = alongs[i];
    }
    if (sums_only) {
      if (threadIdx.x == 0) alongs[i] = r.along;
      continue;
    }
    float along = 0.f;
    if (joins && a.after) {
      for (int64_t j = threadIdx.x * 8; j < a.cols; j += kApart) {
        const int n = columns_left(a.cols, j);
        Eight term;
        const Eight d = stream_gradient<T>(a, r, i, j, n, term), u = RowsOf<T>::get(a.u, i, j, n), w = weight_of(a.v, j, n);
#pragma unroll
        for (int k = 0; k < 8; ++k) along += k < n ? d.v[k] * (u.v[k] * r.after) * w.v[k] : 0.f;
      }
      along = row_sum<16>(along, room[turn][1]) * each;
    }
    for (int64_t j = threadIdx.x * 8; j < a.cols; j += kApart) {
      const int n = columns_left(a.cols, j);
      Eight term;
      const Eight d = stream_gradient<T>(a, r, i, j, n, term);
      Eight du = {};
      if (joins && a.du.base) {
        const Eight w = weight_of(a.v, j, n);
        du = RowsOf<T>::get(a.u, i, j, n);
#pragma unroll
        for (int k = 0; k < 8; ++k) du.v[k] = r.after * (d.v[k] * w.v[k] - du.v[k] * r.after * along);
        put_up_to8<T>(a.du.base, i * a.du.stride + j, n, du);
      }
      if (a.dx.base) {
        Eight dx;
#pragma unroll
        for (int k = 0; k < 8; ++k) dx.v[k] = joins ? a.v.keep * d.v[k] : d.v[k];
        put_up_to8<T>(a.dx.base, i * a.dx.stride + j, n, dx);
      }
    }
  }
}

// Rows of any length: the lines of both sums.  A work-group has 512 columns and every (4 * parts)-th row for each of its wavefronts.
template <typename T>
__global__ __launch_bounds__(256) void ds_join_params_long_kernel(JoinBackward a, const float *alongs) {
  __shared__ float sums[2][4][64][8 + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t j = ((int64_t)blockIdx.x * 64 + lane) * 8;
  const int n = columns_left(a.cols, j);
  Eight da = {}, db = {};
  for (int64_t i = (int64_t)blockIdx.y * 4 + wave; i < a.rows; i += (int64_t)gridDim.y * 4) {
    const LongRow r = {a.before ? a.rstd_before[i] : 0.f, a.after ? a.rstd_after[i] : 1.f, alongs[i]};
    Eight term;
    const Eight d = stream_gradient<T>(a, r, i, j, n, term);
    Eight u = {};
    if (a.u.base) u = RowsOf<T>::get(a.u, i, j, n);
#pragma unroll
    for (int k = 0; k < 8; ++k) da.v[k] += term.v[k], db.v[k] += k < n ? d.v[k] * (u.v[k] * r.after) : 0.f;
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) sums[0][wave][lane][k] = da.v[k], sums[1][wave][lane][k] = db.v[k];
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

// The lines added, and what they are the gradients of.  A work-group has 16 columns (and further ones where a launch has no place for as many
// work-groups), and each of its 16 rows of threads every 16th line; then those 16 sums in their order.  blockIdx.y: a or b.
__global__ __launch_bounds__(256) void ds_join_sums_kernel(const float *partial, int64_t parts, int64_t cols, Vectors v, float *dbefore, float *dgate,
                                                           float *dafter) {
  __shared__ float sums[16][16 + 1];
  const int across = threadIdx.x % 16, row = threadIdx.x / 16;
  if (blockIdx.y ? !dgate && !dafter : !dbefore) return;
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
      if (blockIdx.y == 0) {
        dbefore[j] = s;
      } else {
        if (dgate) dgate[j] = v.scale * s * get_up_to8_any(v.after_gamma, v.dtype, j, 1, 1.f).v[0];
        if (dafter) dafter[j] = v.scale * s * get_up_to8_any(v.gate, v.dtype, j, 1, 1.f).v[0];
      }
    }
    __syncthreads();
  }
}

// Rows of so many columns fit the registers of a work-group.
constexpr int64_t kLongest = 16384, kLongestBackward = 8192;

int64_t join_groups(int64_t rows, int64_t at_a_time, int64_t most) {
  const int64_t sets = (rows + at_a_time - 1) / at_a_time;
  return sets < most ? sets : most;
}

template <typename T>
int launch_forward(const JoinForward &a, hipStream_t stream) {
  const auto launch = [&](auto kernel, int rows, int waves) -> int {
    hipLaunchKernelGGL(kernel, dim3((uint32_t)join_groups(a.rows, rows, 256 * 32 / waves)), dim3(waves * 64), 0, stream, a);
    DS_HIP_TRY(hipGetLastError());
    return DS_OK;
  };
  // few rows: as many wavefronts for each as have something to read
  if (a.rows <= 256 && a.cols > 2048 && a.cols <= 8192) return launch(ds_join_forward_kernel<T, 16, 16, 1>, 1, 16);
  if (a.cols <= 512) return launch(ds_join_forward_kernel<T, 1, 4, 1>, 4, 4);
  if (a.cols <= 2048) return launch(ds_join_forward_kernel<T, 4, 4, 1>, 1, 4);
  if (a.cols <= 4096) return launch(ds_join_forward_kernel<T, 4, 4, 2>, 1, 4);
  if (a.cols <= 8192) return launch(ds_join_forward_kernel<T, 8, 8, 2>, 1, 8);
  if (a.cols <= kLongest) return launch(ds_join_forward_kernel<T, 16, 16, 2, sizeof(T) == 2>, 1, 16);
  return launch(ds_join_forward_long_kernel<T>, 1, 16);
}

int64_t join_parts(int64_t rows, int64_t cols) {
  if (rows <= 0) return 1;
  if (cols <= 512) return join_groups(rows, 4, 512);
  if (cols <= kLongestBackward) return join_groups(rows, 1, 512);
  const int64_t across = (cols + 511) / 512;
  return join_groups(rows, 4, (1024 + across - 1) / across);
}
// The lines, then for long rows one float each.
int64_t join_workspace(int64_t rows, int64_t cols) { return 4 * (2 * join_parts(rows, cols) * cols + (cols > kLongestBackward ? rows : 0)); }

template <typename T>
int launch_backward(const JoinBackward &a, int64_t parts, hipStream_t stream) {
  const auto launch = [&](auto kernel, int waves) -> int {
    hipLaunchKernelGGL(kernel, dim3((uint32_t)parts), dim3(waves * 64), 0, stream, a);
    DS_HIP_TRY(hipGetLastError());
    return DS_OK;
  };
  if (a.cols <= 512) return launch(ds_join_backward_kernel<T, 1, 4, 1>, 4);
  if (a.cols <= 2048) return launch(ds_join_backward_kernel<T, 4, 4, 1>, 4);
  if (a.cols <= 4096) return launch(ds_join_backward_kernel<T, 8, 8, 1>, 8);
  if (a.cols <= kLongestBackward) return launch(ds_join_backward_kernel<T, 16, 16, 1>, 16);
  // the parameters' sums first: dx may be dout
  const dim3 grid((uint32_t)join_groups(a.rows, 1, 4096));
  float *alongs = nullptr;
  if (a.partial) {
    alongs = a.partial + 2 * parts * a.cols;
    hipLaunchKernelGGL(ds_join_backward_long_kernel<T>, grid, dim3(1024), 0, stream, a, alongs, true);
    DS_HIP_TRY(hipGetLastError());
    hipLaunchKernelGGL(ds_join_params_long_kernel<T>, dim3((uint32_t)((a.cols + 511) / 512), (uint32_t)parts), dim3(256), 0, stream, a, alongs);
    DS_HIP_TRY(hipGetLastError());
  }
  if (a.du.base || a.dx.base) {
    hipLaunchKernelGGL(ds_join_backward_long_kernel<T>, grid, dim3(1024), 0, stream, a, alongs, false);
    DS_HIP_TRY(hipGetLastError());
  }
  return DS_OK;
}

int check_join(const ds_join *join) {
  if (!join || join->reserved || (join->norms & ~(DS_JOIN_AFTER | DS_JOIN_BEFORE)) || !ds_is_float(join->param_dtype) || !(join->eps >= 0.f) ||
      (join->after_gamma && !(join->norms & DS_JOIN_AFTER)) || (join->before_gamma && !(join->norms & DS_JOIN_BEFORE)))
    return DS_EINVAL;
  const int size = ds_itemsize(join->param_dtype);
  return ds_misaligned(join->after_gamma, size) || ds_misaligned(join->gate, size) || ds_misaligned(join->before_gamma, size) ? DS_EINVAL : DS_OK;
}

// A matrix of `like`'s type and extents, or none where that is allowed.
int check_like(const ds_matrix *m, const ds_matrix *like, bool needed) {
  if (!m) return needed ? DS_EINVAL : DS_OK;
  DS_TRY(ds_check_matrix(m, true));
  return m->dtype == like->dtype && ds_same_extents(m, like) ? DS_OK : DS_EINVAL;
}

int check_first(const ds_matrix *m) {
  DS_TRY(ds_check_matrix(m, true));
  return m->dtype == DS_MX8 ? DS_EINVAL : DS_OK;
}

Vectors vectors_of(const ds_join *j) {
  return Vectors{j->after_gamma, j->gate, j->before_gamma, j->param_dtype, j->keep, j->scale, j->eps};
}

}  // namespace

extern "C" int ds_join_forward(const ds_join *join, const ds_matrix *u, const ds_matrix *x, const ds_matrix *out, const ds_matrix *y,
                               float *rstd_after, float *rstd_before, void *stream) {
  DS_TRY(check_join(join));
  DS_TRY(check_first(x));
  const bool after = join->norms & DS_JOIN_AFTER, before = join->norms & DS_JOIN_BEFORE;
  DS_TRY(check_like(u, x, false));
  DS_TRY(check_like(out, x, u != nullptr));
  DS_TRY(check_like(y, x, before));
  if ((!u && (out || after || join->gate)) || (!before && y) || (!after && rstd_after) || (!before && rstd_before) || (!u && !before) ||
      ds_misaligned(rstd_after, 4) || ds_misaligned(rstd_before, 4))
    return DS_EINVAL;
  if (x->rows == 0 || x->cols == 0) return DS_OK;
  const JoinForward a{ds_rows(u), ds_rows(x), ds_rows(out), ds_rows(y), vectors_of(join), rstd_after, rstd_before, x->rows, x->cols, after, before};
  return ds_with_type(x->dtype, [&](auto type) -> int { return launch_forward<decltype(type)>(a, (hipStream_t)stream); });
}

extern "C" int ds_join_backward_workspace(int64_t rows, int64_t cols, uint64_t *bytes) {
  if (!bytes || rows < 0 || cols < 0) return DS_EINVAL;
  if (rows > kMaxExtent || cols > kMaxExtent) return DS_ERANGE;
  *bytes = (uint64_t)join_workspace(rows, cols);
  return DS_OK;
}

extern "C" int ds_join_backward(const ds_join *join, const ds_matrix *dout, const ds_matrix *dy, const ds_matrix *u, const ds_matrix *out,
                                const float *rstd_after, const float *rstd_before, const ds_matrix *du, const ds_matrix *dx,
                                float *dafter, float *dgate, float *dbefore, void *workspace, uint64_t workspace_bytes, void *stream) {
  DS_TRY(check_join(join));
  const bool after = join->norms & DS_JOIN_AFTER, before = join->norms & DS_JOIN_BEFORE;
  const ds_matrix *first = dy ? dy : dout;
  DS_TRY(check_first(first));
  DS_TRY(check_like(dout, first, !before));
  DS_TRY(check_like(dy, first, before));
  DS_TRY(check_like(u, first, false));
  DS_TRY(check_like(out, first, before));
  DS_TRY(check_like(du, first, false));
  DS_TRY(check_like(dx, first, false));
  if ((!u && (du || after || join->gate || dgate || dafter)) || (!before && (dy || out || rstd_before || dbefore)) || (!after && (rstd_after || dafter)) ||
      (!u && !before) || ds_misaligned(rstd_after, 4) || ds_misaligned(rstd_before, 4) || ds_misaligned(dafter, 4) || ds_misaligned(dgate, 4) ||
      ds_misaligned(dbefore, 4))
    return DS_EINVAL;
  const int64_t rows = first->rows, cols = first->cols;
  const bool sums = dafter || dgate || dbefore;
  if (cols == 0 || (rows == 0 && !sums)) return DS_OK;
  if (rows > 0 && ((after && !rstd_after) || (before && !rstd_before))) return DS_EINVAL;
  const int64_t parts = join_parts(rows, cols);
  if (sums) {
    if (!workspace || ds_misaligned(workspace, 16)) return DS_EINVAL;
    if (workspace_bytes < (uint64_t)join_workspace(rows, cols)) return DS_ERANGE;
  }
  hipStream_t st = (hipStream_t)stream;
  const JoinBackward a{ds_rows(dout), ds_rows(dy), ds_rows(u), ds_rows(out), ds_rows(du), ds_rows(dx), vectors_of(join), rstd_after, rstd_before,
                       sums ? (float *)workspace : nullptr, rows, cols, after, before};
  if (rows > 0)
    DS_TRY(ds_with_type(first->dtype, [&](auto type) -> int { return launch_backward<decltype(type)>(a, parts, st); }));
  if (!sums) return DS_OK;
  const int64_t groups = (cols + 15) / 16;
  hipLaunchKernelGGL(ds_join_sums_kernel, dim3((uint32_t)(groups < kMaxGrid ? groups : kMaxGrid), 2), dim3(256), 0, st, (const float *)workspace,
                     rows > 0 ? parts : 0, cols, a.v, dbefore, dgate, dafter);
  DS_HIP_TRY(hipGetLastError());
  return DS_OK;
}
