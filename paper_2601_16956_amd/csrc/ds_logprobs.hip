// Log probabilities of tokens: forward, with entropy and the likeliest tokens, and backward.
//
// Both are bound by HBM: forward reads the logits once, backward reads them and writes their gradient.  A row belongs to one
// to sixteen wavefronts, whose threads have pieces of neighbouring columns, 16 bytes each; each thread keeps, of what it has seen, the
// largest logit m, s = sum exp(scale (x - m)) and t = sum exp(scale (x - m)) (x - m), and where m grows it multiplies them
// by exp of the difference (t after the difference times s was added).  Threads' triples are joined by the same rule, in an order
// that only the extents and `top` decide.  Then logsum = log(s) and entropy = logsum - scale t / s.
//
// The likeliest: the largest logit of every piece goes to LDS.  The threads of a row are 64 sets, and the bound is the `top`-th of the sets'
// largest logits: as many columns reach it, so the pieces that reach it contain those wanted, and mostly few others (of logits in any order, 64 log(64 /
// (64 - top)) columns: 24 for 20).  These pieces are read again, an element by each thread, and what reaches the bound is put into LDS, where each is
// ranked by counting those in front of it.
// Columns are in the order of a key of their logit and place, which no two share.  Where more reach the bound than LDS has room for (many
// equal ones, rows in order, few columns that are not masked), the `top`-th of the first 256 found is a higher bound, and it is tried again.
//
// Few rows are cut into parts, one work-group each, whose triples and likeliest a second launch joins.
//
// us, bf16 logits unless said: 8192 x 32000 forward 92 (5.7 TB/s) and backward 176 (6.0 TB/s); 1 x 32000 with five likeliest 7.7; 2048 x 32000 fp16 with ten
// 32 (4.1 TB/s: the search for them, beside which none of its work-group's loads are under way); 37 x 50021 floats with 20 likeliest 7.6 + 4.4;
// 1024 x 1024 floats forward 3.9, backward 4.4, 4096 x 32000 floats 89 (5.9 TB/s) and 165 (6.3 TB/s).

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ds_ops.h"

namespace {

constexpr float kInf = __builtin_inff();
constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kCandidates = 512, kSample = 256;  // room for columns that may be among the likeliest, and for pieces that have such
constexpr int kMostPieces = 8192;                // of a row, or a part, whose likeliest are looked for

struct Triple {
  float m, s, t;
};

// Infinities: m = -infinity is nothing seen, and stands for 0 where it is subtracted.  The product of a factor that is 0 and a
// difference that is infinite is 0: differences are held above the lowest float.  A NaN or +infinity makes s NaN for good.
__device__ inline float finite_or_0(float m) { return m == -kInf ? 0.f : m; }

template <bool ENTROPY>
__device__ inline void raise(Triple &a, float m, float c) {
  const float gap = fmaxf(a.m - finite_or_0(m), kLowest), f = __builtin_amdgcn_exp2f(gap * c);
  if (ENTROPY) a.t = f > 0.f ? f * (a.t + gap * a.s) : 0.f;
  a.s *= f;
  a.m = m;
}
// A piece: 16 bytes, 8 or 4 columns.
template <typename T>
constexpr int kColumns = 16 / (int)sizeof(T);
template <typename T>
struct Piece {
  float v[kColumns<T>];
};
template <typename T>
__device__ inline Piece<T> piece_of(const ds_u32x4 &bits) {
  Piece<T> x;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int k = 0; k < 4; ++k) x.v[k] = __uint_as_float(bits[k]);
  } else {
    const Eight e = Elem<T>::get8(&bits, 0);
#pragma unroll
    for (int k = 0; k < 8; ++k) x.v[k] = e.v[k];
  }
  return x;
}
template <typename T>
__device__ inline ds_u32x4 bits_of(const Piece<T> &x) {
  ds_u32x4 bits;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int k = 0; k < 4; ++k) bits[k] = __float_as_uint(x.v[k]);
  } else {
    Eight e;
#pragma unroll
    for (int k = 0; k < 8; ++k) e.v[k] = x.v[k];
    Elem<T>::put8(&bits, 0, e);
  }
  return bits;
}
// Columns from j on, as many as there are up to `end`; the others are masked.
template <typename T>
__device__ inline Piece<T> piece_at(const T *row, int64_t j, int64_t end) {
  if (j + kColumns<T> <= end) return piece_of<T>(*(const ds_u32x4 *)(row + j));
  Piece<T> x;
#pragma unroll
  for (int k = 0; k < kColumns<T>; ++k) x.v[k] = j + k < end ? Elem<T>::get(row, j + k) : -kInf;
  return x;
}

// Returns the piece's largest logit.
template <typename T, bool ENTROPY>
__device__ inline float add(Triple &a, const Piece<T> &x, float c) {
  float peak = x.v[0];
#pragma unroll
  for (int k = 1; k < kColumns<T>; ++k) peak = fmaxf(peak, x.v[k]);
  const float m = fmaxf(a.m, peak);
  raise<ENTROPY>(a, m, c);
  const float base = finite_or_0(m);
#pragma unroll
  for (int k = 0; k < kColumns<T>; ++k) {
    const float d = x.v[k] - base, e = __builtin_amdgcn_exp2f(d * c);
    a.s += e;
    if (ENTROPY) a.t += e * fmaxf(d, kLowest);
  }
  return peak;
}

// Larger for a larger logit, and of equal ones for the lower column; 0 is below all.
__device__ inline uint64_t key_of(float x, int64_t j) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return (uint64_t)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (0xffffffffu - (uint32_t)j);
}
__device__ inline float key_logit(uint64_t key) {
  const uint32_t b = (uint32_t)(key >> 32);
  return __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b);
}
__device__ inline int64_t key_column(uint64_t key) { return (int64_t)(0xffffffffu - (uint32_t)key); }

struct Forward {
  Rows x;
  const int64_t *tokens;
  float *logprob, *largest, *logsum, *entropy;
  int64_t *top_tokens;
  float *top_logprobs;
  int64_t rows, cols;
  float scale;
  uint32_t top;
  // rows in parts: a part's columns (a multiple of eight), their number, and what they leave
  int64_t part_cols;
  int32_t parts;
  Triple *triples;  // [rows][parts]
  uint64_t *keys;   // [rows][parts][top]
};

__device__ inline int64_t token_of(const Forward &a, int64_t i) {
  const int64_t token = a.tokens ? a.tokens[i] : -1;
  return token >= 0 && token < a.cols ? token : -1;
}
// scale * (x - m).  (A difference of 2^128 or more is no float; its product with a scale below 1 may be.)
__device__ inline float scaled(const Forward &a, float x, float m) { return a.scale < 1.f ? 2.f * a.scale * (0.5f * x - 0.5f * m) : a.scale * (x - m); }
// A row's numbers out of its triple.  `at`: the logit of the token, if there is one.
__device__ inline void put_row(const Forward &a, int64_t i, Triple r, bool given, float at) {
  const bool none = r.m == -kInf && r.s == 0.f;
  const float nan = __uint_as_float(0x7fc00000u), logsum = none ? -kInf : logf(r.s);
  const bool bad = !(r.s < kInf);
  if (a.largest) a.largest[i] = bad ? nan : r.m;
  if (a.logsum) a.logsum[i] = bad ? nan : logsum;
  if (a.entropy) a.entropy[i] = bad ? nan : none ? 0.f : logsum - a.scale * (r.t / r.s);
  if (a.logprob) a.logprob[i] = !given ? 0.f : bad ? nan : at == -kInf ? -kInf : scaled(a, at, r.m) - logsum;
}
__device__ inline void put_top(const Forward &a, int64_t i, int rank, uint64_t key, Triple r) {
  const bool bad = !(r.s < kInf);
  if (a.top_tokens) a.top_tokens[i * a.top + rank] = key && !bad ? key_column(key) : -1;
  if (a.top_logprobs) a.top_logprobs[i * a.top + rank] = bad ? __uint_as_float(0x7fc00000u) : key ? scaled(a, key_logit(key), r.m) - logf(r.s) : -kInf;
}

template <bool ENTROPY>
__device__ inline Triple wave_triple(Triple a, float c) {
  raise<ENTROPY>(a, all_max(a.m), c);
  a.s = all_sum(a.s);
  if (ENTROPY) a.t = all_sum(a.t);
  return a;
}

template <int THREADS>
struct Room {
  Triple triples[THREADS / 64];
  alignas(16) float sets[64];
  alignas(16) float least[4];
  uint64_t keys[kCandidates];
  uint64_t bound;
  uint32_t hits[kCandidates];
  uint16_t threads[THREADS];
  uint32_t n_hits, count;
};

// The row's triple, in every thread.
template <int THREADS, bool ENTROPY>
__device__ inline Triple row_triple(Triple a, float c, Triple *room) {
  a = wave_triple<ENTROPY>(a, c);
  if (THREADS == 64) return a;
  if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = a;
  __syncthreads();
  const int lane = threadIdx.x & 63;
  a = lane < THREADS / 64 ? room[lane] : Triple{-kInf, 0.f, 0.f};
  return wave_triple<ENTROPY>(a, c);
}

// How many of `count` keys are larger.  (Eight at a time are on their way; those behind the last are 0.)
__device__ inline int rank_of(uint64_t key, const uint64_t *keys, int count) {
  int rank = 0;
#pragma unroll 1
  for (int k = 0; k < count; k += 8)
#pragma unroll
    for (int e = 0; e < 8; ++e) rank += keys[k + e] > key;
  return rank;
}

// The same by four neighbouring lanes, each of which compares every fourth eight.
__device__ inline int rank_of_four(uint64_t key, const uint64_t *keys, int count) {
  int rank = 0;
#pragma unroll 1
  for (int k = (threadIdx.x & 3) * 8; k < count; k += 32)
#pragma unroll
    for (int e = 0; e < 8; ++e) rank += keys[k + e] > key;
  rank += __builtin_amdgcn_update_dpp(0, rank, 0xB1, 0xf, 0xf, true);
  return rank + __builtin_amdgcn_update_dpp(0, rank, 0x4E, 0xf, 0xf, true);
}

// The likeliest of `count` columns from row[0] on, handed to put(rank, key) by one thread each.  `m`: the thread's largest logit, `peaks`: its
// pieces' (every THREADS-th); `begin`: the number of the first column.
template <typename T, int THREADS, typename Put>
__device__ inline void likeliest(const T *row, int count, int64_t begin, uint32_t top, float m, const float *peaks, Room<THREADS> &room, Put put) {
  constexpr int W = kColumns<T>;
  const int pieces = (count + W - 1) / W, lane = threadIdx.x & 63;
  const int shift = pieces <= THREADS ? 0 : min(32 - __clz((pieces - 1) / THREADS), 6);  // lanes of a thread's pieces, as a power of two
  const float most = m;
  // threads in 64 sets
  if (THREADS >= 256) m = larger(m, moved<0xB1, 0xf>(m, m)), m = larger(m, moved<0x4E, 0xf>(m, m));
  if (THREADS >= 1024) m = larger(m, moved<0x141, 0xf>(m, m)), m = larger(m, moved<0x140, 0xf>(m, m));
  if (threadIdx.x == 0) room.n_hits = room.count = 0;
  if (threadIdx.x % (THREADS / 64) == 0) room.sets[threadIdx.x / (THREADS / 64)] = m;
  __syncthreads();
  // the `top`-th of the 64, of equal ones the first that so many are not larger than: four lanes a set where there are as many
  float least;
  if (THREADS == 64) {
    const float set = room.sets[lane];
    uint32_t larger_ones = 0;
#pragma unroll
    for (int q = 0; q < 64; ++q) larger_ones += room.sets[q] > set;
    least = -all_max(larger_ones < top ? -set : -kInf);
  } else {
    if (threadIdx.x < 256) {
      const float set = room.sets[threadIdx.x / 4];
      int larger_ones = 0;
#pragma unroll
      for (int q = 0; q < 16; ++q) larger_ones += room.sets[q / 4 * 16 + (threadIdx.x & 3) * 4 + q % 4] > set;
      larger_ones += __builtin_amdgcn_update_dpp(0, larger_ones, 0xB1, 0xf, 0xf, true);
      larger_ones += __builtin_amdgcn_update_dpp(0, larger_ones, 0x4E, 0xf, 0xf, true);
      const float of_wave = all_max(larger_ones < (int)top ? -set : -kInf);
      if (lane == 0) room.least[threadIdx.x / 64] = of_wave;
    }
    __syncthreads();
    least = -larger(larger(room.least[0], room.least[1]), larger(room.least[2], room.least[3]));
  }
  uint64_t bound = least == -kInf ? 1 : key_of(least, 0xffffffff);
  int found;
  for (;;) {
    // Pieces that have a column that reaches the bound, or (one of them) might have: of the threads whose largest logit does, whose pieces the
    // lanes of their wavefront share.
    const bool some = most > -kInf && key_of(most, 0) >= bound;
    const uint64_t mask = __ballot(some);
    if (some) room.threads[threadIdx.x / 64 * 64 + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0))] = (uint16_t)threadIdx.x;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int t = lane >> shift; t < __popcll(mask); t += 64 >> shift)
#pragma unroll 1
      for (int p = room.threads[threadIdx.x / 64 * 64 + t] + (lane & ((1 << shift) - 1)) * THREADS; p < pieces; p += THREADS << shift) {
        const float peak = peaks[p];
        if (!(peak > -kInf && key_of(peak, begin + p * W) >= bound)) continue;
        const uint32_t at = atomicAdd(&room.n_hits, 1u);
        if (at < kCandidates) room.hits[at] = p;
      }
    __syncthreads();
    const int hits = (int)room.n_hits;
#pragma unroll 1
    for (int e = threadIdx.x; e < min(hits, kCandidates) * W; e += 2 * THREADS) {
      float x[2];
      int j[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int of = min(e + u * THREADS, min(hits, kCandidates) * W - 1);
        j[u] = (int)room.hits[of / W] * W + of % W;
        x[u] = Elem<T>::get(row, min(j[u], count - 1));
        if (j[u] >= count || of != e + u * THREADS) x[u] = -kInf;
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint64_t key = key_of(x[u], begin + j[u]);
        if (!(x[u] > -kInf && key >= bound)) continue;
        const uint32_t at = atomicAdd(&room.count, 1u);
        if (at < kCandidates) room.keys[at] = key;
      }
    }
    __syncthreads();
    found = (int)room.count;
    if (hits <= kCandidates && found <= kCandidates) break;
    __syncthreads();
    // a higher bound in every turn: at least kSample columns were found, no two keys are equal, and fewer are wanted
#pragma unroll 1
    for (int at = threadIdx.x; at < kSample; at += THREADS)
      if (rank_of(room.keys[at], room.keys, kSample) == (int)top - 1) room.bound = room.keys[at];
    if (threadIdx.x == 0) room.n_hits = room.count = 0;
    __syncthreads();
    bound = room.bound;
  }
  if (threadIdx.x < 32 && found + threadIdx.x < kCandidates) room.keys[found + threadIdx.x] = 0;
  __syncthreads();
#pragma unroll 1
  for (int at = threadIdx.x / 4; at < found; at += THREADS / 4) {
    const uint64_t key = room.keys[at];
    const int rank = rank_of_four(key, room.keys, found);
    if ((threadIdx.x & 3) == 0 && rank < (int)top) put(rank, key);
  }
  for (int rank = found + threadIdx.x; rank < (int)top; rank += THREADS) put(rank, 0);
}

// What a work-group leaves of its row, or part.
__device__ inline void finish(const Forward &a, int64_t item, int64_t i, Triple r, int64_t token, float at) {
  if (threadIdx.x) return;
  if (a.parts > 1) a.triples[item] = r;
  else put_row(a, i, r, token >= 0, at);
}
__device__ inline void put_likely(const Forward &a, int64_t item, int64_t i, int rank, uint64_t key, Triple r) {
  if (a.parts == 1) put_top(a, i, rank, key, r);
  else a.keys[item * a.top + rank] = key;
}

// A work-group has a row, or a part of one: kAhead pieces of each thread at a time, the next ones on their way.  Every load is made, so that
// none waits for those behind it: a piece that is not whole is the last columns of a piece's size, those that others have masked.  TOP: with
// the likeliest.
constexpr int kAhead = 4;
template <typename T, int THREADS, bool ENTROPY, bool TOP>
__global__ __launch_bounds__(THREADS) void ds_logprobs_kernel(Forward a) {
  __shared__ std::conditional_t<TOP, Room<THREADS>, Triple[THREADS / 64]> room;
  extern __shared__ float peaks[];  // TOP: one for each piece
  Triple *triples = (Triple *)&room;
  constexpr int W = kColumns<T>, kStep = kAhead * THREADS * W;
  const float c = a.scale * kLog2e;
  for (int64_t item = blockIdx.x; item < a.rows * a.parts; item += gridDim.x) {
    const int64_t i = a.parts == 1 ? item : item / a.parts, part = item - i * a.parts;
    const int64_t begin = part * a.part_cols, end = begin + a.part_cols < a.cols ? begin + a.part_cols : a.cols;
    const int count = (int)(end - begin), at = threadIdx.x * W;
    const T *row = (const T *)a.x.base + i * a.x.stride + begin;
    Triple r = {-kInf, 0.f, 0.f};
    const int64_t token = a.parts == 1 && threadIdx.x == 0 ? token_of(a, i) : -1;
    if (count >= W) {
      ds_u32x4 bits[kAhead], next[kAhead];
      const auto ask = [&](int first, ds_u32x4 *to) {
#pragma unroll
        for (int e = 0; e < kAhead; ++e) to[e] = *(const ds_u32x4 *)(row + min(first + e * THREADS * W + at, count - W));
      };
      ask(0, bits);
      for (int first = 0;;) {
        const int left = count - first;
        ask(left > kStep ? first + kStep : first, next);
        if (left >= kStep) {
#pragma unroll
          for (int e = 0; e < kAhead; ++e) {
            const float peak = add<T, ENTROPY>(r, piece_of<T>(bits[e]), c);
            if (TOP) peaks[first / W + e * THREADS + threadIdx.x] = peak;
          }
        } else {
#pragma unroll
          for (int e = 0; e < kAhead; ++e) {
            const int shift = e * THREADS * W + at - (left - W);
            if (shift >= W) break;
            Piece<T> x = piece_of<T>(bits[e]);
#pragma unroll
            for (int k = 0; k < W; ++k) x.v[k] = k >= shift ? x.v[k] : -kInf;
            const float peak = add<T, ENTROPY>(r, x, c);
            if (TOP) peaks[first / W + e * THREADS + threadIdx.x] = peak;
          }
        }
        if (left <= kStep) break;
        first += kStep;
#pragma unroll
        for (int e = 0; e < kAhead; ++e) bits[e] = next[e];
      }
    } else if (at < count) {
      const float peak = add<T, ENTROPY>(r, piece_at(row, at, count), c);
      if (TOP) peaks[threadIdx.x] = peak;
    }
    const float m = r.m, given = token >= 0 ? Elem<T>::get(row, token) : 0.f;
    r = row_triple<THREADS, ENTROPY>(r, c, triples);
    finish(a, item, i, r, token, given);
    if constexpr (TOP)
      likeliest<T, THREADS>(row, count, begin, a.top, m, peaks, room, [&](int rank, uint64_t key) { put_likely(a, item, i, rank, key, r); });
    if (THREADS > 64 || TOP) __syncthreads();
  }
}

// The parts of a row joined: a work-group has a row, of 64 threads, or 1024 with the likeliest.  Those so far, and as many of the parts' as the 256
// places have room for, are ranked by four threads each until all have been.  (37 x 6 parts with 20 each: 4.4 us, by one thread each
// 5.7; 8 parts with 32 each 5.6 and 7.4.)
constexpr int kMostKeys = 256 - (int)DS_TOP_MOST;
template <typename T, bool ENTROPY>
__global__ __launch_bounds__(1024) void ds_logprobs_join_kernel(Forward a) {
  alignas(16) __shared__ uint64_t keys[256];
  __shared__ uint64_t best[DS_TOP_MOST];
  const float c = a.scale * kLog2e;
  for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x) {
    const int lane = threadIdx.x & 63, place = threadIdx.x / 4, quarter = threadIdx.x & 3, spare = place - (int)DS_TOP_MOST;
    const int64_t token = token_of(a, i), count = (int64_t)a.parts * a.top;
    const float at = token >= 0 ? Elem<T>::get(a.x.base, i * a.x.stride + token) : 0.f;
    uint64_t key = spare >= 0 && spare < count ? a.keys[i * count + spare] : 0;
    Triple r = {-kInf, 0.f, 0.f};
    for (int p = lane; p < a.parts; p += 64) {
      Triple o = a.triples[i * a.parts + p];
      const float m = fmaxf(r.m, o.m);
      raise<ENTROPY>(r, m, c), raise<ENTROPY>(o, m, c);
      r.s += o.s, r.t += o.t;
    }
    r = wave_triple<ENTROPY>(r, c);
    if (threadIdx.x == 0) put_row(a, i, r, token >= 0, at);
    if (!a.top) continue;
    for (int64_t first = 0; first < count; first += kMostKeys) {
      __syncthreads();
      if (spare < 0) key = first ? best[place] : 0;
      else if (first) key = first + spare < count ? a.keys[i * count + first + spare] : 0;
      if (quarter == 0) keys[place] = key;
      __syncthreads();
      if (spare < 0) best[place] = 0;
      __syncthreads();
      if (key) {
        const int rank = rank_of_four(key, keys, (int)(count - first < kMostKeys ? count - first : kMostKeys) + (int)DS_TOP_MOST);
        if (quarter == 0 && rank < (int)a.top) best[rank] = key;
      }
    }
    __syncthreads();
    if (threadIdx.x < a.top) put_top(a, i, threadIdx.x, best[threadIdx.x], r);
  }
}

struct Backward {
  Rows x, dx;
  const int64_t *tokens;
  const float *largest, *logsum, *entropy, *dlogprob, *dentropy;
  int64_t rows, cols;
  float scale;
  uint32_t across;  // work-groups of a row
};

// A work-group has kPiecesEach * 256 pieces of a row.  (Loads as above.)
constexpr int kPiecesEach = 4;
template <typename T, bool ENTROPY, bool STREAM>
__global__ __launch_bounds__(256) void ds_logprobs_backward_kernel(Backward a) {
  constexpr int W = kColumns<T>, kStep = kPiecesEach * 256 * W;
  for (int64_t item = blockIdx.x; item < a.rows * a.across; item += gridDim.x) {
    const int64_t i = item / a.across, first = (item - i * a.across) * kStep;
    const int left = (int)(a.cols - first < kStep ? a.cols - first : kStep), at = threadIdx.x * W;
    const T *row = (const T *)a.x.base + i * a.x.stride + first;
    T *to = (T *)a.dx.base + i * a.dx.stride + first;
    // (a piece before the row's end, which may begin before `first`; or, in a row shorter than a piece, none)
    const bool pieces = a.cols >= W;
    ds_u32x4 bits[kPiecesEach] = {};
    if (pieces) {
#pragma unroll
      for (int e = 0; e < kPiecesEach; ++e) {
        const ds_u32x4 *from = (const ds_u32x4 *)(row + min(e * 256 * W + at, left - W));
        bits[e] = STREAM ? __builtin_nontemporal_load(from) : *from;
      }
    }
    const int64_t token = a.tokens ? a.tokens[i] : -1;
    const bool given = token >= 0 && token < a.cols;
    const float up = given && a.dlogprob ? a.dlogprob[i] * a.scale : 0.f, along = ENTROPY ? a.dentropy[i] * a.scale : 0.f;
    const float m = a.largest[i], logsum = a.logsum[i], h = ENTROPY ? a.entropy[i] : 0.f;
    const bool zero = m == -kInf || (up == 0.f && along == 0.f);
    const float c = a.scale * kLog2e, o = logsum * kLog2e;
#pragma unroll
    for (int e = 0; e < kPiecesEach; ++e) {
      const int j = e * 256 * W + at, shift = j - (left - W);
      if (left < kStep && j >= left) break;
      Piece<T> x = {};
      if (!zero) {
        x = pieces ? piece_of<T>(bits[e]) : piece_at(row, j, left);
#pragma unroll
        for (int k = 0; k < W; ++k) {
          const float z = x.v[k] - m, p = __builtin_amdgcn_exp2f(__builtin_fmaf(z, c, -o));
          x.v[k] = ENTROPY ? (p == 0.f ? 0.f : -p * (up + along * (__builtin_fmaf(z, a.scale, -logsum) + h))) : -p * up;
        }
        const int64_t column = token - first - (pieces ? min(j, left - W) : j);
        if (given && column >= 0 && column < W) {
#pragma unroll
          for (int k = 0; k < W; ++k) x.v[k] += column == k ? up : 0.f;
        }
      }
      if (pieces && shift <= 0) {
        const ds_u32x4 o = bits_of<T>(x);
        if (STREAM) __builtin_nontemporal_store(o, (ds_u32x4 *)(to + j));
        else *(ds_u32x4 *)(to + j) = o;
      } else {
#pragma unroll
        for (int k = 0; k < W; ++k) {
          const int column = pieces ? left - W + k : j + k;
          if (column >= j && column < left) Elem<T>::put(to, column, x.v[k]);
        }
      }
    }
  }
}

// Bytes of a gradient from which on its accesses are not temporal: the gradient would leave the caches late, while others read.  So / by ordinary
// accesses, us of the backward pass and the forward pass of the next rows: bf16, 32000 columns, 1024 rows (66 MB) 24 + 16 / 24 + 19, 2048 rows 47 +
// 29 / 45 + 40, 4096 rows 92 + 54 / 89 + 73, 8192 rows 178 + 100 / 177 + 125.
constexpr int64_t kStream = 64 << 20;

// Parts of a row: where few rows of more than kWhole columns leave most of the card idle, so many that the work-groups are about as many as the
// CUs, each of at least kLeast columns, and no more candidates than the kernel that joins them has places; but as many as it takes where the
// likeliest are looked for.  bf16, us of both kernels, whole / in parts of 32768 columns / of 8192: 1 x 32000 with five likeliest 7.0 / - / 9.5,
// 1 x 128000 - / 11.4 / 10.7 and without them 9.5 / 7.3 / 6.7, 16 x 128000 with five - / 13.0 / 12.0, 1 x 500000 without 28.8 / 7.8 / 6.8.
constexpr int64_t kWhole = 32768, kLeast = 8192;
int64_t part_cols_of(int64_t cols, int64_t parts) { return ((cols + parts - 1) / parts + 7) / 8 * 8; }
int64_t parts_of(int64_t rows, int64_t cols, uint32_t top, int64_t size) {
  int64_t parts = 1;
  if (rows <= 128 && cols > kWhole) {
    parts = std::min(256 / rows, (cols + kLeast - 1) / kLeast);
    if (top) parts = std::min<int64_t>(parts, kMostKeys / top);
    parts = std::min<int64_t>(parts, 64);
  }
  const int64_t most = kMostPieces * 16 / size;
  return std::max(parts, top ? (cols + most - 1) / most : 1);
}

uint64_t workspace_of(int64_t rows, int64_t parts, uint32_t top) {
  if (parts == 1) return 0;
  return (uint64_t)(((rows * parts * (int64_t)sizeof(Triple) + 15) & ~15ll) + rows * parts * top * 8);
}

int check_logits(const ds_matrix *x) {
  DS_TRY(ds_check_matrix(x, true));
  return x->dtype == DS_MX8 ? DS_EINVAL : DS_OK;
}

// Its product with log2(e) is finite, and that with a difference of logits which no float holds (2^128 or more: an infinity) would be beyond every
// exponential's range too; sums of differences times their exponentials, each at most 1 / scale, are floats.
bool is_scale(float s) { return s >= 0x1p-64f && s < 0x1p127f; }

}  // namespace

extern "C" int ds_logprobs_workspace(const ds_matrix *logits, uint32_t top, uint64_t *bytes) {
  DS_TRY(check_logits(logits));
  if (!bytes || top > DS_TOP_MOST) return DS_EINVAL;
  const int64_t rows = logits->rows, cols = logits->cols, size = ds_itemsize(logits->dtype);
  *bytes = 0;
  // (enough for a call without the likeliest too)
  if (rows && cols)
    *bytes = std::max(workspace_of(rows, parts_of(rows, cols, top, size), top), workspace_of(rows, parts_of(rows, cols, 0, size), 0));
  return DS_OK;
}

extern "C" int ds_logprobs(const ds_matrix *logits, float scale, const int64_t *tokens, float *logprob, float *largest, float *logsum,
                           float *entropy, uint32_t top, int64_t *top_tokens, float *top_logprobs, void *workspace, uint64_t workspace_bytes,
                           void *stream) {
  DS_TRY(check_logits(logits));
  if (!is_scale(scale) || top > DS_TOP_MOST || (logprob && !tokens) || ds_misaligned(tokens, 8) || ds_misaligned(logprob, 4) ||
      ds_misaligned(largest, 4) || ds_misaligned(logsum, 4) || ds_misaligned(entropy, 4) || ds_misaligned(top_tokens, 8) ||
      ds_misaligned(top_logprobs, 4))
    return DS_EINVAL;
  const int64_t rows = logits->rows, cols = logits->cols;
  if (rows == 0) return DS_OK;
  if (!top_tokens && !top_logprobs) top = 0;
  const int64_t parts = cols ? parts_of(rows, cols, top, ds_itemsize(logits->dtype)) : 1;
  if (parts > 1) {
    if (!workspace || ds_misaligned(workspace, 16)) return DS_EINVAL;
    if (workspace_bytes < workspace_of(rows, parts, top)) return DS_ERANGE;
  }
  const int64_t keys_at = (rows * parts * (int64_t)sizeof(Triple) + 15) & ~15ll, part_cols = part_cols_of(cols, parts);
  const Forward a{ds_rows(logits), tokens, logprob, largest, logsum, entropy, top_tokens, top_logprobs, rows, cols, scale, top, part_cols,
                  (int32_t)parts, (Triple *)workspace, (uint64_t *)((uint8_t *)workspace + keys_at)};
  return ds_with_type(logits->dtype, [&](auto type) -> int {
    typedef decltype(type) T;
    const auto with = [&](auto wanted) -> int {
      constexpr bool E = decltype(wanted)::value;
      const int64_t pieces = top ? (part_cols + kColumns<T> - 1) / kColumns<T> : 0;
      const auto launch = [&](auto kernel, int threads, int64_t groups, int64_t floats) -> int {
        hipLaunchKernelGGL(kernel, dim3((uint32_t)std::min(groups, kMaxGrid)), dim3(threads), (uint32_t)(floats * 4), (hipStream_t)stream, a);
        DS_HIP_TRY(hipGetLastError());
        return DS_OK;
      };
      const auto rows_with = [&](auto likeliest) -> int {
        constexpr bool TOP = decltype(likeliest)::value;
        // One wavefront a row, four, or sixteen.  bf16, us: 4096 rows of 1024 columns 5.0 / 9.2 / -, of 4096 9.3 / 11.9 / -, of 8192 14.9 / 15.0 /
        // -; 64 rows of 2048 3.3 / - / 4.0; 200 rows of 32000 - / 6.5 / 6.4, 300 rows - / 8.2 / 10.2.  With five to twenty likeliest: 4096 rows of 2048 9.8 /
        // 21 / -, of 8192 21.2 / 25.0 / -, of 16000 44 / 38 / -; 3000 rows of 8000 18.1 / 21.5 / -, 1024 rows of 8192 9.2 / 8.8 / -; 512 rows of
        // 32000 - / 12.2 / 17.4.
        const int64_t bytes = cols * (int64_t)sizeof(T);
        if (parts == 1 && bytes <= (rows > 2048 ? 16384 : rows > 256 ? 8192 : 4096)) return launch(ds_logprobs_kernel<T, 64, E, TOP>, 64, rows, pieces);
        if (rows * parts > 256) return launch(ds_logprobs_kernel<T, 256, E, TOP>, 256, rows * parts, pieces);
        return launch(ds_logprobs_kernel<T, 1024, E, TOP>, 1024, rows * parts, pieces);
      };
      DS_TRY(top ? rows_with(std::true_type()) : rows_with(std::false_type()));
      return parts == 1 ? DS_OK : launch(ds_logprobs_join_kernel<T, E>, top ? 1024 : 64, rows, 0);
    };
    return entropy ? with(std::true_type()) : with(std::false_type());
  });
}

extern "C" int ds_logprobs_backward(const ds_matrix *logits, float scale, const int64_t *tokens, const float *largest, const float *logsum,
                                    const float *entropy, const float *dlogprob, const float *dentropy, const ds_matrix *dlogits, void *stream) {
  DS_TRY(check_logits(logits));
  DS_TRY(check_logits(dlogits));
  if (!is_scale(scale) || dlogits->dtype != logits->dtype || !ds_same_extents(logits, dlogits) || (dlogprob && !tokens) || (dentropy && !entropy) ||
      ds_misaligned(tokens, 8) || ds_misaligned(largest, 4) || ds_misaligned(logsum, 4) || ds_misaligned(entropy, 4) || ds_misaligned(dlogprob, 4) ||
      ds_misaligned(dentropy, 4))
    return DS_EINVAL;
  if (logits->rows == 0 || logits->cols == 0) return DS_OK;
  if (!largest || !logsum) return DS_EINVAL;
  const int64_t size = ds_itemsize(logits->dtype), step = kPiecesEach * 256 * 16 / size;
  const uint32_t across = (uint32_t)((logits->cols + step - 1) / step);
  const bool stream_it = logits->rows * logits->cols >= kStream / size;
  const Backward a{ds_rows(logits), ds_rows(dlogits), tokens, largest, logsum, entropy, dlogprob, dentropy, logits->rows, logits->cols, scale, across};
  return ds_with_type(logits->dtype, [&](auto type) -> int {
    typedef decltype(type) T;
    const auto launch = [&](auto kernel) -> int {
      hipLaunchKernelGGL(kernel, dim3((uint32_t)std::min(a.rows * across, kMaxGrid)), dim3(256), 0, (hipStream_t)stream, a);
      DS_HIP_TRY(hipGetLastError());
      return DS_OK;
    };
    if (dentropy) return stream_it ? launch(ds_logprobs_backward_kernel<T, true, true>) : launch(ds_logprobs_backward_kernel<T, true, false>);
    return stream_it ? launch(ds_logprobs_backward_kernel<T, false, true>) : launch(ds_logprobs_backward_kernel<T, false, false>);
  });
}
