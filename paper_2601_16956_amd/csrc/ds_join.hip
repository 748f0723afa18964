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
//
// us, bf16, both norms and a gate: 8192 x 4096 forward 47 (5.7 TB/s), backward 73 + 4.7 for the lines (5.5 TB/s for the first); 1 x 8192 forward
// 4.3; 1537 x 1000 fp16, one norm, backward 11.5 + 3.9.  Floats, 8192 x 2048: forward 52 (5.2 TB/s), backward 82 + 4.7 (4.9 TB/s: no row is on its
// way during another, whose 32-bit words fill the registers).

#include <type_traits>

#include "ds_ops.h"

namespace {

__device__ inline int columns_left(int64_t cols, int64_t j) {
  const int64_t left = cols - j;
  return (int)(left < 0 ? 0 : left < 8 ? left : 8);
}

// Of rows of any length: the sum of `x` over the work-group's wavefronts, in every thread, by `room` as total_of_row does.
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

// Waits for loads here, where what was asked for behind them is known: at the head of a loop the compiler would wait for all.
template <typename B>
__device__ inline void arrived(B &bits) {
#pragma unroll
  for (int q = 0; q < (int)(sizeof(B) / 16); ++q)
#pragma unroll
    for (int k = 0; k < 4; ++k) asm volatile("" : "+v"(bits.w[q][k]));
}

// Eight elements of a row; STREAM: not temporal, where a wavefront's are 1 KiB without a gap.
template <typename T, bool STREAM>
__device__ inline typename RowsOf<T>::Bits ask_eight(const Rows &m, int64_t i, int64_t j) {
  if constexpr (STREAM && sizeof(T) == 2) {
    typename RowsOf<T>::Bits b;
    b.w[0] = __builtin_nontemporal_load((const ds_u32x4 *)((const T *)m.base + i * m.stride + j));
    return b;
  } else {
    return RowsOf<T>::ask(m, i, j, 8);
  }
}
template <typename T, bool STREAM>
__device__ inline void put_eight(const Rows &m, int64_t i, int64_t j, const Eight &x) {
  if constexpr (STREAM && sizeof(T) == 2) {
    ds_u32x4 bits;
    Elem<T>::put8(&bits, 0, x);
    __builtin_nontemporal_store(bits, (ds_u32x4 *)((T *)m.base + i * m.stride + j));
  } else {
    Elem<T>::put8(m.base, i * m.stride + j, x);
  }
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

// The sum of a row's `WAVES` wavefronts, the which-th of the work-group, in every thread.  `room`: a float for each wavefront, another one in
// every turn: it is written again only behind the barrier of a sum in between.
template <int WAVES>
__device__ inline float total_of_row(float x, float *room, int which) {
  x = all_sum(x);
  if (WAVES == 1) return x;
  if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = x;
  __syncthreads();
  x = room[which * WAVES + threadIdx.x % WAVES];
  x += moved<0xB1, 0xf>(x, 0.f);
  if (WAVES >= 4) x += moved<0x4E, 0xf>(x, 0.f);
  if (WAVES >= 8) x += moved<0x141, 0xf>(x, 0.f);
  if (WAVES >= 16) x += moved<0x140, 0xf>(x, 0.f);
  return x;
}

// WAVES wavefronts have a row, each thread HAS pieces of it, 512 * WAVES columns apart; a work-group of WIDE wavefronts has WIDE / WAVES rows at a
// time, and the next ones on their way.  The compiler counts what is on its way only where nothing is conditional, and waits for all of it,
// the last row's stores too, elsewhere.  So, from a row of a piece on (PIECES), every load and store is made: a piece that is not whole is the row's
// last eight columns, left out of the sums where others have them, but computed and stored as they do; rows beyond the last are the last;
// without a block x is read for u.  Nothing is stored before the whole row has been read: out may be x.
template <typename T, int WAVES, int WIDE, int HAS, bool PIECES, bool STREAM>
__global__ __launch_bounds__(WIDE * 64) void ds_join_forward_kernel(JoinForward a) {
  __shared__ float room[2][2][WIDE];
  constexpr int kRows = WIDE / WAVES, kApart = WAVES * 512;
  const int at = threadIdx.x % (WAVES * 64) * 8, which = kRows == 1 ? 0 : threadIdx.x / (WAVES * 64);
  const bool joins = a.u.base != nullptr;
  const Rows u_or_x = joins ? a.u : a.x;
  const float each = 1.f / (float)a.cols;
  const int64_t stride = (int64_t)gridDim.x * kRows;
  int n[HAS], from[HAS], others[HAS];
  Eight w[HAS], g[HAS];
#pragma unroll
  for (int p = 0; p < HAS; ++p) {
    const int j = at + p * kApart;
    n[p] = columns_left(a.cols, j);
    from[p] = PIECES && n[p] < 8 ? (int)a.cols - 8 : j, others[p] = j - from[p];
    w[p] = weight_of(a.v, from[p], PIECES ? 8 : n[p]);
    g[p] = get_up_to8_any(a.v.before_gamma, a.v.dtype, from[p], PIECES ? 8 : n[p], 1.f);
  }
  typedef typename RowsOf<T>::Bits Bits;
  Bits next_x[HAS], next_u[HAS];
  const auto ask = [&](int64_t i) {
    const int64_t there = i < a.rows ? i : a.rows - 1;
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
      next_x[p] = PIECES ? ask_eight<T, STREAM>(a.x, there, from[p]) : RowsOf<T>::ask(a.x, there, from[p], n[p]);
      next_u[p] = PIECES ? ask_eight<T, STREAM>(u_or_x, there, from[p]) : RowsOf<T>::ask(u_or_x, there, from[p], n[p]);
    }
  };
  const auto put = [&](const Rows &to, int64_t i, int p, const Eight &x) {
    const int64_t there = i < a.rows ? i : a.rows - 1;
    if (PIECES) put_eight<T, STREAM>(to, there, from[p], x);
    else put_up_to8<T>(to.base, there * to.stride + from[p], n[p], x);
  };
  constexpr bool kAhead = sizeof(T) == 2 || HAS == 1;  // where the registers hold both rows
  int64_t i = (int64_t)blockIdx.x * kRows + which;
  if (kAhead) ask(i);
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.rows; first += stride, i += stride, turn ^= 1) {
    if (!kAhead) ask(i);
    Eight x[HAS], u[HAS];
    float squares = 0.f;
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
      x[p] = RowsOf<T>::value(next_x[p], 8), u[p] = RowsOf<T>::value(next_u[p], 8);
#pragma unroll
      for (int k = 0; k < 8; ++k) squares += k >= others[p] ? u[p].v[k] * u[p].v[k] : 0.f;
    }
    if (kAhead) ask(first + stride < a.rows ? i + stride : i);
    float after = 1.f;
    if (a.after) after = 1.f / sqrtf(total_of_row<WAVES>(squares, room[turn][0], which) * each + a.v.eps);
    squares = 0.f;
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
      if (joins) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[p].v[k] = a.v.keep * x[p].v[k] + u[p].v[k] * after * w[p].v[k];
        as_stored<T>(x[p]);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) squares += k >= others[p] ? x[p].v[k] * x[p].v[k] : 0.f;
    }
    const float before = 1.f / sqrtf(total_of_row<WAVES>(squares, room[turn][1], which) * each + a.v.eps);
    if (WAVES == 1) __syncthreads();
    if (at == 0 && i < a.rows) {
      if (a.after && a.rstd_after) a.rstd_after[i] = after;
      if (a.before && a.rstd_before) a.rstd_before[i] = before;
    }
#pragma unroll
    for (int p = 0; p < HAS; ++p) {
      if (joins) put(a.out, i, p, x[p]);
      if (!a.before) continue;
#pragma unroll
      for (int k = 0; k < 8; ++k) x[p].v[k] = x[p].v[k] * before * g[p].v[k];
      put(a.y, i, p, x[p]);
    }
    if (kAhead) {
#pragma unroll
      for (int p = 0; p < HAS; ++p) arrived(next_x[p]), arrived(next_u[p]);
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

// WAVES wavefronts have a row, each thread a piece of it; a work-group of WIDE wavefronts has WIDE / WAVES rows at a time, and the next ones on
// their way.  The norms' sums are taken together: with A = sum g h / cols,
//   sum w k = sum (scale gate after_gamma) k (dout + rstd_before g) - rstd_before A sum (scale gate after_gamma) k h.
// The compiler counts what is on its way only where nothing is conditional, and waits for all of it, the last row's stores too, elsewhere.  So, from
// a row of a piece on (PIECES), every load and store is made: a piece that is not whole is the row's last eight columns, left out of the
// sums where others have them, but computed and stored as they do; rows beyond the last are the last; what there is none of is read from
// where there is something.  WHOLE: all pieces are whole and the threads' own.  BOTH: du and dx are wanted.
template <typename T, int WAVES, int WIDE, bool PIECES, bool WHOLE, bool BOTH, bool STREAM>
__global__ __launch_bounds__(WIDE * 64) void ds_join_backward_kernel(JoinBackward a) {
  constexpr int kRows = WIDE / WAVES, kApart = WAVES * 512;
  __shared__ float room[2][3][WIDE];
  __shared__ float lines[kRows > 1 ? kRows : 1][kRows > 1 ? kApart : 1];
  const int at = threadIdx.x % (WAVES * 64) * 8, which = kRows == 1 ? 0 : threadIdx.x / (WAVES * 64);
  const bool joins = a.u.base != nullptr;
  JoinBackward s = a;
  if (PIECES) {
    const Rows some = a.before ? a.dy : a.dout;
    if (!a.dout.base) s.dout = some;
    if (!a.before) s.dy = s.out = some, s.rstd_before = (const float *)some.base;
    if (!joins) s.u = some;
    if (!a.after) s.rstd_after = (const float *)some.base;
  }
  const float each = 1.f / (float)a.cols;
  const int64_t stride = (int64_t)gridDim.x * kRows;
  const int n = WHOLE ? 8 : columns_left(a.cols, at);
  const int from = PIECES && n < 8 ? (int)a.cols - 8 : at, others = at - from;  // the first column, and how many are others'
  const Eight g = get_up_to8_any(a.v.before_gamma, a.v.dtype, from, PIECES ? 8 : n, 1.f), w = weight_of(a.v, from, PIECES ? 8 : n);
  Eight da = {}, db = {};
  struct Row {
    typename RowsOf<T>::Bits d, u, y, o;
    float before, after;
  };
  const auto ask = [&](Row &r, int64_t i) {
    const int64_t there = i < a.rows ? i : a.rows - 1;
    if (PIECES) {
      r.d = ask_eight<T, STREAM>(s.dout, there, from), r.u = ask_eight<T, STREAM>(s.u, there, from);
      r.y = ask_eight<T, STREAM>(s.dy, there, from), r.o = ask_eight<T, STREAM>(s.out, there, from);
      r.before = s.rstd_before[there], r.after = s.rstd_after[there];
      return;
    }
    r = Row{};
    if (a.dout.base) r.d = RowsOf<T>::ask(a.dout, there, from, n);
    if (a.before) r.y = RowsOf<T>::ask(a.dy, there, from, n), r.o = RowsOf<T>::ask(a.out, there, from, n), r.before = a.rstd_before[there];
    if (joins) r.u = RowsOf<T>::ask(a.u, there, from, n);
    if (a.after) r.after = a.rstd_after[there];
  };
  const auto put = [&](const Rows &to, int64_t i, const Eight &x) {
    const int64_t there = i < a.rows ? i : a.rows - 1;
    if (PIECES) put_eight<T, STREAM>(to, there, from, x);
    else put_up_to8<T>(to.base, there * to.stride + from, n, x);
  };
  int64_t i = (int64_t)blockIdx.x * kRows + which;
  constexpr bool kAhead = sizeof(T) == 2;  // rows of 32 bits fill the registers as it is
  Row next;
  if (kAhead) ask(next, i);
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.rows; first += stride, i += stride, turn ^= 1) {
    if (!kAhead) ask(next, i);
    const Row now = next;
    if (kAhead) ask(next, first + stride < a.rows ? i + stride : i);
    const float before = a.before ? now.before : 0.f, after = a.after ? now.after : 1.f;
    // (chosen by it, not multiplied with it: a row may have infinities; the wavefront's lanes have one row)
    const bool counts = kRows == 1 || __builtin_amdgcn_readfirstlane((int)(i < a.rows));
    Eight d = RowsOf<T>::value(now.d, 8), k = RowsOf<T>::value(now.u, 8), y = RowsOf<T>::value(now.y, 8), h = RowsOf<T>::value(now.o, 8);
    float sum[3] = {};
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      d.v[c] = a.dout.base ? d.v[c] : 0.f;
      y.v[c] = a.before ? y.v[c] : 0.f, h.v[c] = a.before ? h.v[c] * before : 0.f;
      k.v[c] = joins ? k.v[c] * after : 0.f;
      da.v[c] += counts ? y.v[c] * h.v[c] : 0.f;
      y.v[c] *= g.v[c];
      d.v[c] += before * y.v[c];
      const bool own = WHOLE || c >= others;
      const float wk = own ? w.v[c] * k.v[c] : 0.f;
      sum[0] += own ? y.v[c] * h.v[c] : 0.f, sum[1] += wk * d.v[c], sum[2] += wk * h.v[c];
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) sum[q] = all_sum(sum[q]);
    // (rows beyond the last are computed and stored as the last is: all have read it before one writes, as dx may be dout)
    if (WAVES == 1) __syncthreads();
    if (WAVES > 1) {
      if ((threadIdx.x & 63) < 3) room[turn][threadIdx.x & 63][threadIdx.x >> 6] = (threadIdx.x & 63) == 0 ? sum[0] : (threadIdx.x & 63) == 1 ? sum[1] : sum[2];
      __syncthreads();
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        float x = room[turn][q][which * WAVES + threadIdx.x % WAVES];
        x += moved<0xB1, 0xf>(x, 0.f);
        if (WAVES >= 4) x += moved<0x4E, 0xf>(x, 0.f);
        if (WAVES >= 8) x += moved<0x141, 0xf>(x, 0.f);
        if (WAVES >= 16) x += moved<0x140, 0xf>(x, 0.f);
        sum[q] = x;
      }
    }
    const float flow = before * (sum[0] * each), along = a.after ? (sum[1] - flow * sum[2]) * each : 0.f;
    Eight du;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      d.v[c] -= flow * h.v[c];
      db.v[c] += counts ? d.v[c] * k.v[c] : 0.f;
      du.v[c] = after * (d.v[c] * w.v[c] - (a.after ? k.v[c] * along : 0.f));  // (without the norm u, which may be no number, is nothing to du)
      d.v[c] *= joins ? a.v.keep : 1.f;
    }
    if (BOTH || a.du.base) put(a.du, i, du);
    if (BOTH || a.dx.base) put(a.dx, i, d);
    if (kAhead) {
      arrived(next.d), arrived(next.u), arrived(next.y), arrived(next.o);
      asm volatile("" : "+v"(next.before), "+v"(next.after));
    }
  }
  if (!a.partial) return;
  const int64_t parts = gridDim.x;
  const auto put_line = [&](int s, const Eight &x) {
    float *to = a.partial + (s * parts + blockIdx.x) * a.cols;
    if (n >= 8) return put_up_to8<float>(to, at, 8, x);
#pragma unroll
    for (int c = 0; c < 8; ++c)
      if (c >= others && from + c < a.cols) to[from + c] = x.v[c];
  };
  if (kRows == 1) {
    put_line(0, da), put_line(1, db);
    return;
  }
  // the rows' wavefronts are added in their order
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    __syncthreads();
#pragma unroll
    for (int c = 0; c < 8; ++c)
      if (c >= others && from + c < a.cols) lines[which][from + c] = s ? db.v[c] : da.v[c];
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
        if (a.after) du = RowsOf<T>::get(a.u, i, j, n);
#pragma unroll
        for (int k = 0; k < 8; ++k) du.v[k] = r.after * (d.v[k] * w.v[k] - du.v[k] * r.after * along);  // (without the norm du and `along` are 0)
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

// Rows of so many columns fit the registers of a work-group: two matrices of them forward, four backward.  us, bf16, on either side of it: forward 2048 x 16384
// 52 (5.1 TB/s), 2048 x 20000, whose second and third passes read again, 101 (3.2); backward 4096 x 8192 74 + 7 (5.0), 2048 x 16384, in three launches
// that read a matrix two or three times, 43 + 43 + 113 + 5 (2.0).
constexpr int64_t kLongest = 16384, kLongestBackward = 8192;

int64_t join_groups(int64_t rows, int64_t at_a_time, int64_t most) {
  const int64_t sets = (rows + at_a_time - 1) / at_a_time;
  return sets < most ? sets : most;
}

// Bytes that a call moves from which on its accesses are not temporal: no cache holds them until someone else reads them.  So / by ordinary
// accesses, us, bf16, rows of 4096: forward 8192 rows (268 MB) 47.4 / 52.9, 2048 rows (67 MB) 15.6 / 14.5; backward with the lines' sums 8192 rows (403 MB)
// 77.1 / 85.5, 2048 rows (101 MB) 30.6 / 29.8.
constexpr int64_t kStream = 256 << 20;
template <typename T>
bool streams(int64_t elements) {
  return sizeof(T) == 2 && elements >= kStream / 2;
}

template <typename T>
int launch_forward(const JoinForward &a, hipStream_t stream) {
  const auto launch = [&](auto kernel, int rows, int waves) -> int {
    hipLaunchKernelGGL(kernel, dim3((uint32_t)join_groups(a.rows, rows, 256 * 16 / waves)), dim3(waves * 64), 0, stream, a);
    DS_HIP_TRY(hipGetLastError());
    return DS_OK;
  };
  if (a.cols < 8) return launch(ds_join_forward_kernel<T, 1, 8, 1, false, false>, 8, 8);
  const auto of_width = [&](auto streams) -> int {
    constexpr bool STREAM = decltype(streams)::value;
    if (a.cols <= 512) return launch(ds_join_forward_kernel<T, 1, 8, 1, true, STREAM>, 8, 8);
    if (a.cols <= 1024) return launch(ds_join_forward_kernel<T, 2, 8, 1, true, STREAM>, 4, 8);
    if (a.cols <= 2048) return launch(ds_join_forward_kernel<T, 4, 8, 1, true, STREAM>, 2, 8);
    if (a.cols <= 4096) return launch(ds_join_forward_kernel<T, 8, 8, 1, true, STREAM>, 1, 8);
    if (a.cols <= 8192) return launch(ds_join_forward_kernel<T, 16, 16, 1, true, STREAM>, 1, 16);
    return launch(ds_join_forward_kernel<T, 16, 16, 2, true, STREAM>, 1, 16);
  };
  if (a.cols <= kLongest) return streams<T>(4 * a.rows * a.cols) ? of_width(std::integral_constant<bool, sizeof(T) == 2>()) : of_width(std::false_type());
  return launch(ds_join_forward_long_kernel<T>, 1, 16);
}

int64_t join_parts(int64_t rows, int64_t cols) {
  if (rows <= 0) return 1;
  // work-groups of 16 wavefronts, one on each CU: as many lines as that takes
  if (cols <= kLongestBackward) return join_groups(rows, cols <= 512 ? 16 : cols <= 1024 ? 8 : cols <= 2048 ? 4 : cols <= 4096 ? 2 : 1, 256);
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
  const auto of_width = [&](auto waves) -> int {
    constexpr int kWaves = decltype(waves)::value;
    constexpr bool S = sizeof(T) == 2;
    const bool whole = kWaves > 1 && a.cols == kWaves * 512;
    if (!a.du.base || !a.dx.base) return launch(ds_join_backward_kernel<T, kWaves, 16, true, false, false, false>, 16);
    if (streams<T>(6 * a.rows * a.cols))
      return whole ? launch(ds_join_backward_kernel<T, kWaves, 16, true, kWaves != 1, true, S>, 16)
                   : launch(ds_join_backward_kernel<T, kWaves, 16, true, false, true, S>, 16);
    return whole ? launch(ds_join_backward_kernel<T, kWaves, 16, true, kWaves != 1, true, false>, 16)
                 : launch(ds_join_backward_kernel<T, kWaves, 16, true, false, true, false>, 16);
  };
  if (a.cols < 8) return launch(ds_join_backward_kernel<T, 1, 16, false, false, false, false>, 16);
  if (a.cols <= 512) return of_width(std::integral_constant<int, 1>());
  if (a.cols <= 1024) return of_width(std::integral_constant<int, 2>());
  if (a.cols <= 2048) return of_width(std::integral_constant<int, 4>());
  if (a.cols <= 4096) return of_width(std::integral_constant<int, 8>());
  if (a.cols <= kLongestBackward) return of_width(std::integral_constant<int, 16>());
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
