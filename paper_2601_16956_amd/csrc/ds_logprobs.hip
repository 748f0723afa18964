// Log probabilities of tokens: forward, with entropy and the likeliest tokens, and backward.
//
// Both are bound by HBM: forward reads the logits once, backward reads them and writes their gradient.  A row belongs to one
// to sixteen wavefronts, whose threads have pieces of eight neighbouring columns; each thread keeps, of what it has seen, the
// largest logit m, s = sum exp(scale (x - m)) and t = sum exp(scale (x - m)) (x - m), and where m grows it multiplies them
// by exp of the difference (t after the difference times s was added).  Threads' triples are joined by the same rule, in an order
// that only the row's length decides.  Then logsum = log(s) and entropy = logsum - scale t / s.
//
// The likeliest: the lanes of a row are 64 sets; the `top`-th largest of the sets' largest logits is one that at least `top` columns
// reach, so the columns that reach it contain those wanted, and mostly few others.  The threads that have such columns read theirs
// again, out of the caches, and put them into LDS, where each is ranked by counting those in front of it.  Columns are in the
// order of a key of their logit and place, which no two share.  Where more columns reach the bound than LDS has room for
// (many equal ones, or few columns that are not masked), the row is read once for each rank instead.
//
// Few rows are cut into parts, one work-group each, whose triples and likeliest a second launch joins.

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ds_ops.h"

namespace {

constexpr float kInf = __builtin_inff();
constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kCandidates = 1024;

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
template <bool ENTROPY>
__device__ inline Triple join(Triple a, Triple b, float c) {
  const float m = fmaxf(a.m, b.m);
  raise<ENTROPY>(a, m, c), raise<ENTROPY>(b, m, c);
  return {m, a.s + b.s, a.t + b.t};
}
template <bool ENTROPY>
__device__ inline void add8(Triple &a, const Eight &x, float c) {
  float m = a.m;
#pragma unroll
  for (int k = 0; k < 8; ++k) m = fmaxf(m, x.v[k]);
  raise<ENTROPY>(a, m, c);
  const float base = finite_or_0(m);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float d = x.v[k] - base, e = __builtin_amdgcn_exp2f(d * c);
    a.s += e;
    if (ENTROPY) a.t += e * fmaxf(d, kLowest);
  }
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
// A row's numbers out of its triple.  `at`: the logit of the token, if there is one.
__device__ inline void put_row(const Forward &a, int64_t i, Triple r, bool given, float at) {
  const bool none = r.m == -kInf && r.s == 0.f;
  const float nan = __uint_as_float(0x7fc00000u), logsum = none ? -kInf : logf(r.s);
  const bool bad = !(r.s < kInf);
  if (a.largest) a.largest[i] = bad ? nan : r.m;
  if (a.logsum) a.logsum[i] = bad ? nan : logsum;
  if (a.entropy) a.entropy[i] = bad ? nan : none ? 0.f : logsum - a.scale * (r.t / r.s);
  if (a.logprob) a.logprob[i] = !given ? 0.f : bad ? nan : at == -kInf ? -kInf : a.scale * (at - r.m) - logsum;
}
__device__ inline void put_top(const Forward &a, int64_t i, int rank, uint64_t key, Triple r) {
  const bool bad = !(r.s < kInf);
  if (a.top_tokens) a.top_tokens[i * a.top + rank] = key && !bad ? key_column(key) : -1;
  if (a.top_logprobs) a.top_logprobs[i * a.top + rank] = bad ? __uint_as_float(0x7fc00000u) : key ? a.scale * (key_logit(key) - r.m) - logf(r.s) : -kInf;
}

__device__ inline uint64_t wave_max(uint64_t x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const uint64_t o = __shfl_xor((unsigned long long)x, d, 64);
    x = o > x ? o : x;
  }
  return x;
}

template <int THREADS>
struct Room {
  Triple triples[THREADS / 64];
  float sets[64];
  uint64_t keys[kCandidates];
  uint64_t best[THREADS / 64];
  uint32_t count;
};

// The row's triple, in every thread.
template <int THREADS, bool ENTROPY>
__device__ inline Triple row_triple(Triple a, float c, Triple *room) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) a = join<ENTROPY>(a, {__shfl_xor(a.m, d, 64), __shfl_xor(a.s, d, 64), __shfl_xor(a.t, d, 64)}, c);
  if (THREADS == 64) return a;
  if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = a;
  __syncthreads();
  a = room[0];
  for (int w = 1; w < THREADS / 64; ++w) a = join<ENTROPY>(a, room[w], c);
  return a;
}

// The likeliest of the columns from `begin` to `end`, handed to put(rank, key) by one thread each; `m`: the thread's largest logit.
template <typename T, int THREADS, typename Put>
__device__ inline void likeliest(const Forward &a, int64_t i, int64_t begin, int64_t end, float m, Room<THREADS> &room, Put put) {
  // the sets' largest, and the `top`-th of those
  for (int d = 1; d < THREADS / 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
  if (threadIdx.x == 0) room.count = 0;
  if (threadIdx.x % (THREADS / 64) == 0) room.sets[threadIdx.x / (THREADS / 64)] = m;
  __syncthreads();
  const float set = room.sets[threadIdx.x & 63];
  int before = 0;
  for (int k = 0; k < 64; ++k) {
    const float other = room.sets[k];
    before += other > set || (other == set && k < (int)(threadIdx.x & 63));
  }
  const uint64_t here = __ballot(before == (int)a.top - 1);
  const float bound = __shfl(set, __builtin_ctzll(here | 1ull << 63), 64);
  if (m >= bound && m > -kInf) {
    for (int64_t j = begin + threadIdx.x * 8; j < end; j += THREADS * 8) {
      const int n = (int)(end - j < 8 ? end - j : 8);
      const Eight x = RowsOf<T>::get(a.x, i, j, n);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < n && x.v[k] >= bound && x.v[k] > -kInf) {
          const uint32_t at = atomicAdd(&room.count, 1u);
          if (at < kCandidates) room.keys[at] = key_of(x.v[k], j + k);
        }
    }
  }
  __syncthreads();
  const uint32_t count = room.count;
  if (count <= kCandidates) {
    for (uint32_t at = threadIdx.x; at < count; at += THREADS) {
      const uint64_t key = room.keys[at];
      uint32_t rank = 0;
      for (uint32_t k = 0; k < count; ++k) rank += room.keys[k] > key;
      if (rank < a.top) put((int)rank, key);
    }
    for (uint32_t rank = count + threadIdx.x; rank < a.top; rank += THREADS) put((int)rank, 0);
    return;
  }
  uint64_t last = ~0ull;
  for (uint32_t rank = 0; rank < a.top; ++rank) {
    uint64_t best = 0;
    for (int64_t j = begin + threadIdx.x * 8; j < end; j += THREADS * 8) {
      const int n = (int)(end - j < 8 ? end - j : 8);
      const Eight x = RowsOf<T>::get(a.x, i, j, n);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint64_t key = key_of(x.v[k], j + k);
        if (k < n && x.v[k] > -kInf && key < last && key > best) best = key;
      }
    }
    best = wave_max(best);
    if (THREADS > 64) {
      __syncthreads();
      if ((threadIdx.x & 63) == 0) room.best[threadIdx.x >> 6] = best;
      __syncthreads();
      for (int w = 0; w < THREADS / 64; ++w) best = room.best[w] > best ? room.best[w] : best;
    }
    if (threadIdx.x == 0) put((int)rank, best);
    last = best ? best : 1;  // behind the last there is none
  }
}

// What is read beyond a row is masked.
template <typename T>
__device__ inline Eight logits_of(const typename RowsOf<T>::Bits &b, int n) {
  Eight x = RowsOf<T>::value(b, n);
  if (n < 8) {
#pragma unroll
    for (int k = 0; k < 8; ++k) x.v[k] = k < n ? x.v[k] : -kInf;
  }
  return x;
}

// A work-group has a row, or a part of one.
template <typename T, int THREADS, bool ENTROPY>
__global__ __launch_bounds__(THREADS) void ds_logprobs_kernel(Forward a) {
  __shared__ Room<THREADS> room;
  constexpr int kAhead = 4;
  const float c = a.scale * kLog2e;
  for (int64_t item = blockIdx.x; item < a.rows * a.parts; item += gridDim.x) {
    const int64_t i = a.parts == 1 ? item : item / a.parts, part = item - i * a.parts;
    const int64_t begin = part * a.part_cols, end = begin + a.part_cols < a.cols ? begin + a.part_cols : a.cols;
    Triple r = {-kInf, 0.f, 0.f};
    for (int64_t first = begin; first < end; first += kAhead * THREADS * 8) {
      typename RowsOf<T>::Bits bits[kAhead];
      int n[kAhead];
#pragma unroll
      for (int e = 0; e < kAhead; ++e) {
        const int64_t j = first + (e * THREADS + threadIdx.x) * 8, left = end - j;
        n[e] = (int)(left < 0 ? 0 : left < 8 ? left : 8);
        bits[e] = RowsOf<T>::ask(a.x, i, j, n[e]);
      }
#pragma unroll
      for (int e = 0; e < kAhead; ++e)
        if (n[e] > 0) add8<ENTROPY>(r, logits_of<T>(bits[e], n[e]), c);
    }
    const float m = r.m;
    r = row_triple<THREADS, ENTROPY>(r, c, room.triples);
    if (a.parts == 1) {
      if (threadIdx.x == 0) {
        const int64_t token = token_of(a, i);
        put_row(a, i, r, token >= 0, token >= 0 ? Elem<T>::get(a.x.base, i * a.x.stride + token) : 0.f);
      }
      if (a.top) likeliest<T, THREADS>(a, i, begin, end, m, room, [&](int rank, uint64_t key) { put_top(a, i, rank, key, r); });
    } else {
      if (threadIdx.x == 0) a.triples[item] = r;
      if (a.top) likeliest<T, THREADS>(a, i, begin, end, m, room, [&](int rank, uint64_t key) { a.keys[item * a.top + rank] = key; });
    }
    if (THREADS > 64 || a.top) __syncthreads();
  }
}

// The parts of a row joined: a work-group has a row.
template <typename T, bool ENTROPY>
__global__ __launch_bounds__(256) void ds_logprobs_join_kernel(Forward a) {
  __shared__ uint64_t keys[kCandidates];
  const float c = a.scale * kLog2e;
  for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x) {
    Triple r = a.triples[i * a.parts];
    for (int p = 1; p < a.parts; ++p) r = join<ENTROPY>(r, a.triples[i * a.parts + p], c);
    if (threadIdx.x == 0) {
      const int64_t token = token_of(a, i);
      put_row(a, i, r, token >= 0, token >= 0 ? Elem<T>::get(a.x.base, i * a.x.stride + token) : 0.f);
    }
    if (!a.top) continue;
    const int count = a.parts * (int)a.top;
    __syncthreads();
    for (int k = threadIdx.x; k < count; k += 256) keys[k] = a.keys[i * count + k];
    __syncthreads();
    // (keys of 0, of parts that have fewer, are behind all others in the order of their place)
    for (int at = threadIdx.x; at < count; at += 256) {
      const uint64_t key = keys[at];
      int rank = 0;
      for (int k = 0; k < count; ++k) rank += keys[k] > key || (keys[k] == key && k < at);
      if (rank < (int)a.top) put_top(a, i, rank, key, r);
    }
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

// A work-group has kPiecesEach * 256 pieces of eight columns of a row.
constexpr int kPiecesEach = 4;
template <typename T>
__global__ __launch_bounds__(256) void ds_logprobs_backward_kernel(Backward a) {
  for (int64_t item = blockIdx.x; item < a.rows * a.across; item += gridDim.x) {
    const int64_t i = item / a.across, first = (item - i * a.across) * (kPiecesEach * 256 * 8);
    typename RowsOf<T>::Bits bits[kPiecesEach];
    int n[kPiecesEach];
#pragma unroll
    for (int e = 0; e < kPiecesEach; ++e) {
      const int64_t j = first + (e * 256 + threadIdx.x) * 8, left = a.cols - j;
      n[e] = (int)(left < 0 ? 0 : left < 8 ? left : 8);
      bits[e] = RowsOf<T>::ask(a.x, i, j, n[e]);
    }
    const int64_t token = a.tokens ? a.tokens[i] : -1;
    const bool given = token >= 0 && token < a.cols;
    const float up = given && a.dlogprob ? a.dlogprob[i] * a.scale : 0.f, along = a.dentropy ? a.dentropy[i] * a.scale : 0.f;
    const float m = a.largest[i], logsum = a.logsum[i], h = a.dentropy ? a.entropy[i] : 0.f;
    const bool zero = m == -kInf || (up == 0.f && along == 0.f);
#pragma unroll
    for (int e = 0; e < kPiecesEach; ++e) {
      const int64_t j = first + (e * 256 + threadIdx.x) * 8;
      Eight x = RowsOf<T>::value(bits[e], n[e]);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float logp = a.scale * (x.v[k] - m) - logsum, p = __builtin_amdgcn_exp2f(logp * kLog2e);
        float d = p == 0.f ? 0.f : -p * (up + along * (logp + h));
        if (given && j + k == token) d += up;
        x.v[k] = zero ? 0.f : d;
      }
      put_up_to8<T>(a.dx.base, i * a.dx.stride + j, n[e], x);
    }
  }
}

// Parts of a row, where few rows leave most of the card idle: so many that the work-groups are about as many as the CUs, each of at least
// kLeast columns; and no more candidates than the kernel that joins them has room for.
constexpr int64_t kLeast = 8192;
int64_t parts_of(int64_t rows, int64_t cols, uint32_t top) {
  if (rows <= 0 || rows > 128) return 1;
  int64_t parts = std::min((256 + rows - 1) / rows, (cols + kLeast - 1) / kLeast);
  if (top) parts = std::min<int64_t>(parts, kCandidates / top);
  return std::max<int64_t>(1, std::min<int64_t>(parts, 64));
}

uint64_t workspace_of(int64_t rows, int64_t cols, uint32_t top) {
  const int64_t parts = parts_of(rows, cols, top);
  if (parts == 1) return 0;
  return (uint64_t)(((rows * parts * (int64_t)sizeof(Triple) + 15) & ~15ll) + rows * parts * top * 8);
}

int check_logits(const ds_matrix *x) {
  DS_TRY(ds_check_matrix(x, true));
  return x->dtype == DS_MX8 ? DS_EINVAL : DS_OK;
}

bool is_scale(float s) { return s > 0.f && s < kInf; }

}  // namespace

extern "C" int ds_logprobs_workspace(const ds_matrix *logits, uint32_t top, uint64_t *bytes) {
  DS_TRY(check_logits(logits));
  if (!bytes || top > DS_TOP_MOST) return DS_EINVAL;
  *bytes = logits->cols ? workspace_of(logits->rows, logits->cols, top) : 0;
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
  const int64_t parts = cols ? parts_of(rows, cols, top) : 1;
  if (parts > 1) {
    if (!workspace || ds_misaligned(workspace, 16)) return DS_EINVAL;
    if (workspace_bytes < workspace_of(rows, cols, top)) return DS_ERANGE;
  }
  const int64_t keys_at = (rows * parts * (int64_t)sizeof(Triple) + 15) & ~15ll, part_cols = ((cols + parts - 1) / parts + 7) / 8 * 8;
  const Forward a{ds_rows(logits), tokens, logprob, largest, logsum, entropy, top_tokens, top_logprobs, rows, cols, scale, top, part_cols,
                  (int32_t)parts, (Triple *)workspace, (uint64_t *)((uint8_t *)workspace + keys_at)};
  return ds_with_type(logits->dtype, [&](auto type) -> int {
    typedef decltype(type) T;
    const auto with = [&](auto wanted) -> int {
      constexpr bool E = decltype(wanted)::value;
      const auto launch = [&](auto kernel, int threads, int64_t groups) -> int {
        hipLaunchKernelGGL(kernel, dim3((uint32_t)std::min(groups, kMaxGrid)), dim3(threads), 0, (hipStream_t)stream, a);
        DS_HIP_TRY(hipGetLastError());
        return DS_OK;
      };
      if (parts == 1 && cols <= 2048) return launch(ds_logprobs_kernel<T, 64, E>, 64, rows);
      if (parts == 1 && rows > 256) return launch(ds_logprobs_kernel<T, 256, E>, 256, rows);
      DS_TRY(launch(ds_logprobs_kernel<T, 1024, E>, 1024, rows * parts));
      return parts == 1 ? DS_OK : launch(ds_logprobs_join_kernel<T, E>, 256, rows);
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
  const uint32_t across = (uint32_t)((logits->cols + kPiecesEach * 2048 - 1) / (kPiecesEach * 2048));
  const Backward a{ds_rows(logits), ds_rows(dlogits), tokens, largest, logsum, entropy, dlogprob, dentropy, logits->rows, logits->cols, scale, across};
  return ds_with_type(logits->dtype, [&](auto type) -> int {
    typedef decltype(type) T;
    hipLaunchKernelGGL(ds_logprobs_backward_kernel<T>, dim3((uint32_t)std::min(a.rows * across, kMaxGrid)), dim3(256), 0, (hipStream_t)stream, a);
    DS_HIP_TRY(hipGetLastError());
    return DS_OK;
  });
}
