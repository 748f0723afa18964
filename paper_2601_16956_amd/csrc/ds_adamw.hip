// AdamW over the tensors of a table, and the sum of the squares of their gradients.
//
// Both are bound by HBM: an element with float parameter and moments and bf16 gradient and copy moves 28 bytes in the step (12 + 2 read, 12 + 2
// written), one with a bf16 parameter and moments in 8 bits 10.1, and 2 in the sum of squares.  The table cuts every tensor into chunks of 2048
// elements.  Where a tensor lies as one row, a chunk's record holds all that is needed of the tensor, so that a work-group is one load by scalars away
// from its data; tensors of rows apart are taken by quads of a row, with a division for each.  A thread has kEach quads, a work-group's width apart, whose
// data are all on their way before the first is computed on.  Moments in 8 bits are in groups of 32 columns, which eight neighbouring lanes hold.
// What tensors have in common (types, kind of moments, whether they are one row) is a kernel's template, and a launch has the chunks of one kind.
//
// A chunk for each work-group: the card takes the next one where one ends.  A loop over chunks with the next one's data on their way was no
// faster, and eight neighbouring elements a thread, whose accesses of 32 bits leave gaps, took 374 to 430 us against 277 in a copy that is streamed
// as the update is.
//
// What all elements share -- 1 - beta^t, the factor of clipping -- is computed from device memory, so that a captured graph
// takes another step whenever it is replayed: in every work-group, by one wavefront each, while the data come.
//
// us, of the step and of the sum of squares: 2.4 M elements in 29 tensors, float moments, bf16 gradients and copies (28 bytes in the step) 11 and
// 5.3; 54.7 M such in one tensor 255 (6.0 TB/s) and 23; 135.8 M with moments in 8 bits (16.1 bytes) 357 (6.1 TB/s) and 52; 2000 tensors of 1 to
// 65536 elements, 11 M in all, float gradients and moments in 8 bits 38.  54.7 M in one tensor whose rows of 4096 lie apart, float moments 287 (5.3 TB/s) and 45, in
// 8 bits 163 (5.4 TB/s) and 41.

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <new>
#include <type_traits>
#include <utility>
#include <vector>

#include "ds_ops.h"

namespace {

constexpr int kThreads = 256;
constexpr int kEach = 2;                       // quads of a thread
constexpr int64_t kQuads = kThreads * kEach;   // of a chunk
// Elements of a table from which on accesses are not temporal: its state is not to stay in the caches, and nothing else that does is to leave.
// A smaller one's may still be there when the next step comes.  Not temporal / ordinary, us of the step alone, with three tables in turn, then with twelve, whose
// states no cache holds: float moments 1 M 6.2 / 6.7, 6.4 / 6.9; 3 M 16.2 / 13.6, 16.6 / 19.9; 6 M 30 / 28, 31 / 36; 8 M 40 / 44, 40 / 46; 17 M 83 / 91; 55 M
// 269 / 294; moments in 8 bits 1 M 6.1 / 6.4, 6.4 / 7.0; 6 M 21.5 / 19.5, 21.4 / 24.7; 12 M 36.5 / 38.0; 25 M 69 / 77; 136 M 360 / 404.  (1 M elements are
// mostly latency, and either way within half a microsecond.)
constexpr int64_t kStream = 8 << 20;
constexpr int64_t kMostElements = 1ll << 37;   // of a table: more than any device holds with two moments; sizes that are a mistake fill no memory with chunks
constexpr int64_t kSquareGroups = 2048;        // work-groups of the sum of squares, for each kind of tensors
constexpr int kSquareChunks = 4;               // chunks that they have on their way at a time

// A tensor in the table.  Its matrices are one row where that is how they lie; their strides are then not looked at.
struct Tensor {
  Rows param, grad, m, v, copy;
  int64_t rows, cols, quads;  // quads of a row: a multiple of eight where moments have 8 bits
  uint32_t number, copy_dtype;
  float decay, rate;
};
struct Chunk {
  int64_t quad;  // the first one
  uint32_t tensor, reserved;
};
// A chunk of a tensor that is one row, with all that is needed of the tensor: one load away from the data.
struct Flat {
  void *param, *grad, *m, *v, *copy;  // of its first element
  uint8_t *m_scale, *v_scale;
  int32_t left;  // elements
  uint32_t at;   // its first element's number
  uint32_t number, copy_dtype;
  float decay, rate;
};
// A kind of tensors: their types, whether they are one row, and their chunks.
struct Kind {
  uint32_t param, grad, eight, flat;
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

// What all elements share.
struct Now {
  float rate;      // settings'
  float step;      // 1 / (1 - beta1^t)
  float root;      // 1 / sqrt(1 - beta2^t)
  uint32_t key;    // mix(t + mix(seed))
  float grad;      // what a gradient is multiplied with
  uint32_t still;  // nothing is to change
};

// By one wavefront each, into `w`.  beta^t - 1 is off by as much of itself as t log(beta), its argument, is at most.
__device__ inline void now_of_step(const Settings &s, Now &w) {
  const int64_t at = *s.step, t = at < 1 ? 1 : at;
  w.rate = s.rate_now ? *s.rate_now : (float)s.rate;
  w.key = mix((uint32_t)t + s.seed);
  w.step = -1.f / expm1f((float)((double)t * s.log_beta1));
  w.root = 1.f / sqrtf(-expm1f((float)((double)t * s.log_beta2)));
}
__device__ inline void now_of_gradients(const Settings &s, Now &w) {
  w.still = 0;
  double c = s.grad_scale;
  if (s.squares) {
    const double sum = *s.squares, norm = sqrt(sum) * fabs(s.grad_scale);
    w.still = !(sum < (double)INFINITY);
    if (s.most_norm > 0.0 && norm > s.most_norm) c = c * s.most_norm / norm;
  }
  w.grad = (float)c;
}

// An address that comes out of a table is one of global memory; the compiler knows that of arguments only, and would otherwise use flat
// accesses, which wait for the scalar loads too.
template <typename T>
__device__ inline T *global(T *p) {
  return (T *)(__attribute__((address_space(1))) T *)(uintptr_t)p;
}
__device__ inline Rows rows_of(const Rows &r) { return Rows{global(r.base), r.stride, global(r.scale), r.scale_stride}; }

// Four neighbouring elements: a wavefront's access of 32-bit elements is then 1 KiB without a gap, which non-temporal accesses need.
struct Four {
  float v[4];
};
typedef uint32_t u32x2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x1 __attribute__((aligned(1)));
template <typename T>
struct QuadOf;
template <>
struct QuadOf<float> {
  typedef uint32_t Bits __attribute__((ext_vector_type(4)));
  typedef u32x4 Memory;
  typedef uint32_t One;
  static __device__ inline Bits one(uint32_t x, int k) { Bits b = {0, 0, 0, 0}; b[k] = x; return b; }
  static __device__ inline uint32_t part(const Bits &b, int k) { return b[k]; }
  static __device__ inline Four value(const Bits &b) { return Four{{__uint_as_float(b[0]), __uint_as_float(b[1]), __uint_as_float(b[2]), __uint_as_float(b[3])}}; }
  static __device__ inline Bits bits(const Four &x) { return Bits{__float_as_uint(x.v[0]), __float_as_uint(x.v[1]), __float_as_uint(x.v[2]), __float_as_uint(x.v[3])}; }
};
struct QuadOfHalves {
  typedef uint32_t Bits __attribute__((ext_vector_type(2)));
  typedef u32x2 Memory;
  typedef uint16_t One;
  static __device__ inline Bits one(uint32_t x, int k) { Bits b = {0, 0}; b[k / 2] = x << (16 * (k % 2)); return b; }
  static __device__ inline uint32_t part(const Bits &b, int k) { return b[k / 2] >> (16 * (k % 2)) & 0xffffu; }
};
template <>
struct QuadOf<__hip_bfloat16> : QuadOfHalves {
  static __device__ inline Four value(const Bits &b) {
    return Four{{__uint_as_float(b[0] << 16), __uint_as_float(b[0] & 0xffff0000u), __uint_as_float(b[1] << 16), __uint_as_float(b[1] & 0xffff0000u)}};
  }
  static __device__ inline Bits bits(const Four &x) {
    return Bits{float_to_bf16(x.v[0]) | float_to_bf16(x.v[1]) << 16, float_to_bf16(x.v[2]) | float_to_bf16(x.v[3]) << 16};
  }
};
template <>
struct QuadOf<__half> : QuadOfHalves {
  static __device__ inline Four value(const Bits &b) {
    return Four{{f16_to_float(b[0] & 0xffffu), f16_to_float(b[0] >> 16), f16_to_float(b[1] & 0xffffu), f16_to_float(b[1] >> 16)}};
  }
  static __device__ inline Bits bits(const Four &x) {
    return Bits{float_to_f16(x.v[0]) | float_to_f16(x.v[1]) << 16, float_to_f16(x.v[2]) | float_to_f16(x.v[3]) << 16};
  }
};
template <>
struct QuadOf<uint8_t> {  // codes
  typedef uint32_t Bits;
  typedef u32x1 Memory;
  typedef uint8_t One;
  static __device__ inline Bits one(uint32_t x, int k) { return x << (8 * k); }
  static __device__ inline uint32_t part(const Bits &b, int k) { return b >> (8 * k) & 255u; }
};
// The first n <= 4 of the four from element `at` on; the others are 0, or not written.  STREAM: not temporal.
template <typename T, bool STREAM>
__device__ inline typename QuadOf<T>::Bits ask_quad(const void *base, int64_t at, int n) {
  typedef QuadOf<T> Q;
  typename Q::Bits b = {};
  const typename Q::One *from = (const typename Q::One *)base + at;
  if (n >= 4) return STREAM ? __builtin_nontemporal_load((const typename Q::Memory *)from) : *(const typename Q::Memory *)from;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k < n) b |= Q::one(from[k], k);
  return b;
}
template <typename T, bool STREAM>
__device__ inline void put_quad(void *base, int64_t at, int n, const typename QuadOf<T>::Bits &b) {
  typedef QuadOf<T> Q;
  typename Q::One *to = (typename Q::One *)base + at;
  if (n >= 4) {
    if (STREAM) __builtin_nontemporal_store((typename Q::Memory)b, (typename Q::Memory *)to);
    else *(typename Q::Memory *)to = b;
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k < n) to[k] = (typename Q::One)Q::part(b, k);
}

// Where quad `item` of a tensor of rows is: its row, its first column, and how many columns of it are there.
__device__ inline void place_of(const Tensor &t, int64_t item, int64_t &i, int64_t &j, int &n) {
  if (t.rows * t.quads <= 0xffffffffll - kQuads) i = (uint32_t)item / (uint32_t)t.quads, j = (uint32_t)item - (uint32_t)i * (uint32_t)t.quads;
  else i = item / t.quads, j = item - i * t.quads;
  j *= 4;
  const int64_t left = i < t.rows ? t.cols - j : 0;
  n = (int)(left < 0 ? 0 : left < 4 ? left : 4);
}
// The largest of eight neighbouring lanes', which hold a group of 32.
__device__ inline uint32_t max_of_eight_lanes(uint32_t m) {
  m = max_of_four_lanes(m);
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xf, 0xf, true);  // the other half of eight, mirrored
  return o > m ? o : m;
}

// sqrt(x) to a unit of the last place.  (The instruction takes no subnormal numbers.)
__device__ inline float root_of(float x) {
  const bool small = x < 0x1p-96f;
  const float r = __builtin_amdgcn_sqrtf(small ? x * 0x1p64f : x);
  return small ? r * 0x1p-32f : r;
}

// param, m and v (before they are rounded) after the step.
__device__ inline void step_of(const Settings &s, const Now &w, float step, float decay, const Four &grad, Four &param, Four &first, Four &second) {
  {
    // rounded after each operation, so that a code, which the last bit may decide, is what the formula in 32 bits says anywhere
#pragma clang fp contract(off)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float x = grad.v[k] * w.grad;
      first.v[k] = first.v[k] * s.beta1 + x * s.rest1;
      second.v[k] = second.v[k] * s.beta2 + x * x * s.rest2;
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    param.v[k] -= decay * param.v[k] + step * first.v[k] * __builtin_amdgcn_rcpf(root_of(second.v[k]) * w.root + s.eps);
}

// Moments in 8 bits, and back, rounded at random: `at` is the number of the first of the four.  All lanes take part; `n`: how many there are.
__device__ inline Four first_of(uint32_t codes, uint32_t scale) {
  const float step = mx8_step(scale);
  Four x;
#pragma unroll
  for (int k = 0; k < 4; ++k) x.v[k] = (float)((int)(codes << (24 - 8 * k)) >> 24) * step;
  return x;
}
__device__ inline Four second_of(uint32_t codes, uint32_t scale) {
  const float none = scale == 255u ? __uint_as_float(0x7fc00000u) : 0.f;
  codes = scale == 255u ? 0u : codes;
  Four x;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t c = codes >> (8 * k) & 255u;
    x.v[k] = c ? __uint_as_float((c << 20) + (scale << 23)) : none;
  }
  return x;
}
__device__ inline void codes_of(const Four &first, const Four &second, uint32_t at, uint32_t &code_m, uint32_t &scale_m, uint32_t &code_v, uint32_t &scale_v) {
  uint32_t top_m = 0, top_v = 0, bits[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    bits[k] = __float_as_uint(second.v[k]);
    top_m = max(top_m, __float_as_uint(first.v[k]) & 0x7fffffffu), top_v = max(top_v, bits[k]);
  }
  scale_m = mx8_scale(max_of_eight_lanes(top_m)), scale_v = uf8_scale(max_of_eight_lanes(top_v));
  const bool tiny = scale_m < 6u;  // 1 / step is no float: the values are made larger first
  const float steps = __uint_as_float((tiny ? 229u - scale_m : 260u - (scale_m == 255u ? 133u : scale_m)) << 23), before = tiny ? 0x1p31f : 1.f;
  const uint32_t base = scale_v << 23;
  const int most = min(255, 2039 - 8 * (int)scale_v);
  uint32_t q[4], c[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t r = mix(at + k);
    const float u = __builtin_fmaf((float)(r & 0xffffu), 0x1p-16f, 0x1p-17f);
    q[k] = (uint32_t)(int)__builtin_amdgcn_fmed3f(__builtin_floorf(__builtin_fmaf(first.v[k] * before, steps, u)), -127.f, 127.f);
    // (what is 0 stays 0: the sum is then below a step, and below 0 where there is a base)
    c[k] = (uint32_t)min(max((int)(bits[k] + (r >> 12 & 0xffff0u) + 8u - base) >> 20, (int)min(bits[k], 1u)), most);
  }
  const uint32_t low = __builtin_amdgcn_perm(q[1], q[0], 0x0c0c0400u), high = __builtin_amdgcn_perm(q[3], q[2], 0x04000c0cu);
  code_m = (low | high) & (scale_m == 255u ? 0u : ~0u);
  code_v = (c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24) & (scale_v == 255u ? 0u : ~0u);
}

// Where four elements are, from the bases on.
struct Place {
  int64_t param, grad, m, v, copy, m_scale, v_scale;
  uint32_t at;  // their number in the tensor
  int n;        // how many of them there are
  bool first;   // of their group
};
template <int FULL>
__device__ inline Place place_flat(uint32_t quad, int left, uint32_t at) {
  const uint32_t j = quad * 4;
  const int more = left - (int)j;
  return Place{j, j, j, j, j, j / kGroup, j / kGroup, at + j, FULL ? 4 : more < 0 ? 0 : more < 4 ? more : 4, j % kGroup == 0};
}
__device__ inline Place place_rows(const Tensor &t, int64_t item) {
  int64_t i, j;
  int n;
  place_of(t, item, i, j, n);
  return Place{i * t.param.stride + j, i * t.grad.stride + j, i * t.m.stride + j, i * t.v.stride + j, i * t.copy.stride + j, i * t.m.scale_stride + j / kGroup,
               i * t.v.scale_stride + j / kGroup, (uint32_t)(i * t.cols + j), n, j % kGroup == 0};
}

// A chunk.  FULL: all its quads are whole.
template <typename P, typename G, bool EIGHT, bool FLAT, bool STREAM, bool FULL>
__device__ inline void step_chunk(const Tensor &t, int64_t quad, int left, const Settings &s, Now &shared, bool begins) {
  typedef std::conditional_t<EIGHT, uint8_t, float> M;
  Place at[kEach];
  typename QuadOf<P>::Bits p[kEach];
  typename QuadOf<G>::Bits g[kEach];
  typename QuadOf<M>::Bits m[kEach], v[kEach];
  uint32_t m_scale[kEach], v_scale[kEach];
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    if (FLAT) at[e] = place_flat<FULL>(e * kThreads + threadIdx.x, left, (uint32_t)quad * 4);
    else at[e] = place_rows(t, quad + e * kThreads + threadIdx.x);
    const Place &o = at[e];
    p[e] = ask_quad<P, STREAM>(t.param.base, o.param, o.n), g[e] = ask_quad<G, STREAM>(t.grad.base, o.grad, o.n);
    m[e] = ask_quad<M, STREAM>(t.m.base, o.m, o.n), v[e] = ask_quad<M, STREAM>(t.v.base, o.v, o.n);
    if (EIGHT) m_scale[e] = o.n > 0 ? t.m.scale[o.m_scale] : 0u, v_scale[e] = o.n > 0 ? t.v.scale[o.v_scale] : 0u;
  }
  if (begins) {
    if (threadIdx.x / 64 == 0) now_of_step(s, shared);
    if (threadIdx.x / 64 == 1) now_of_gradients(s, shared);
    __syncthreads();
  }
  const Now w = shared;
  if (w.still) return;
  const float rate = w.rate * t.rate, step = rate * w.step, decay = rate * t.decay;
  const uint32_t key = mix(t.number + w.key);
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const Place &o = at[e];
    Four x = QuadOf<P>::value(p[e]), first, second;
    if constexpr (EIGHT) first = first_of(m[e], m_scale[e]), second = second_of(v[e], v_scale[e]);
    else first = QuadOf<float>::value(m[e]), second = QuadOf<float>::value(v[e]);
    if (EIGHT && !FULL) {  // a step of NaN is not to reach the places beyond the row
#pragma unroll
      for (int k = 0; k < 4; ++k) first.v[k] = k < o.n ? first.v[k] : 0.f, second.v[k] = k < o.n ? second.v[k] : 0.f;
    }
    step_of(s, w, step, decay, QuadOf<G>::value(g[e]), x, first, second);
    put_quad<P, STREAM>(t.param.base, o.param, o.n, QuadOf<P>::bits(x));
    if (t.copy.base) {
      if (t.copy_dtype == DS_BF16) put_quad<__hip_bfloat16, STREAM>(t.copy.base, o.copy, o.n, QuadOf<__hip_bfloat16>::bits(x));
      else if (t.copy_dtype == DS_F16) put_quad<__half, STREAM>(t.copy.base, o.copy, o.n, QuadOf<__half>::bits(x));
      else put_quad<float, STREAM>(t.copy.base, o.copy, o.n, QuadOf<float>::bits(x));
    }
    if constexpr (EIGHT) {
      uint32_t code_m, code_v, scale_m, scale_v;
      codes_of(first, second, o.at + key, code_m, scale_m, code_v, scale_v);
      put_quad<uint8_t, STREAM>(t.m.base, o.m, o.n, code_m);
      put_quad<uint8_t, STREAM>(t.v.base, o.v, o.n, code_v);
      if (o.n > 0 && o.first) t.m.scale[o.m_scale] = (uint8_t)scale_m, t.v.scale[o.v_scale] = (uint8_t)scale_v;
    } else {
      put_quad<float, STREAM>(t.m.base, o.m, o.n, QuadOf<float>::bits(first));
      put_quad<float, STREAM>(t.v.base, o.v, o.n, QuadOf<float>::bits(second));
    }
  }
}

// A work-group takes a chunk, or several where a launch has no place for as many work-groups.  What it needs of the table is in scalar registers
// before anything is written that the table might be.
template <typename P, typename G, bool EIGHT, bool STREAM>
__global__ __launch_bounds__(kThreads, 6) void ds_adamw_flat_kernel(const Flat *__restrict__ chunks, int64_t count, Settings s) {
  __shared__ Now shared;
  for (int64_t c = blockIdx.x; c < count; c += gridDim.x) {
    const Flat f = chunks[c];
    const auto row = [](void *base, uint8_t *scale) { return Rows{global(base), 0, global(scale), 0}; };
    const Tensor t{row(f.param, nullptr), row(f.grad, nullptr), row(f.m, f.m_scale), row(f.v, f.v_scale), row(f.copy, nullptr), 1, f.left, 0,
                   f.number, f.copy_dtype, f.decay, f.rate};
    const bool begins = c == blockIdx.x;
    if (f.left == kQuads * 4) step_chunk<P, G, EIGHT, true, STREAM, true>(t, f.at / 4, f.left, s, shared, begins);
    else step_chunk<P, G, EIGHT, true, STREAM, false>(t, f.at / 4, f.left, s, shared, begins);
  }
}
template <typename P, typename G, bool EIGHT>
__global__ __launch_bounds__(kThreads) void ds_adamw_rows_kernel(const Tensor *__restrict__ tensors, const Chunk *__restrict__ chunks, int64_t count, Settings s) {
  __shared__ Now shared;
  for (int64_t c = blockIdx.x; c < count; c += gridDim.x) {
    const Chunk chunk = chunks[c];
    Tensor t = tensors[chunk.tensor];
    t.param = rows_of(t.param), t.grad = rows_of(t.grad), t.m = rows_of(t.m), t.v = rows_of(t.v), t.copy = rows_of(t.copy);
    step_chunk<P, G, EIGHT, false, false, false>(t, chunk.quad, 0, s, shared, c == blockIdx.x);
  }
}

__device__ inline double wave_sum(double x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d, 64);
  return x;
}

// One sum for each work-group, in the order of its chunks.  (In 64 bits: gradients' squares span more than 32 bits' exponents do, and the
// sums of ranks are added.)
template <typename G>
__device__ inline void add_squares(const typename QuadOf<G>::Bits &g, double &sum) {
  const Four x = QuadOf<G>::value(g);
#pragma unroll
  for (int k = 0; k < 4; ++k) sum += (double)x.v[k] * (double)x.v[k];
}
__device__ inline void put_sum(double sum, double *partial) {
  __shared__ double sums[kThreads / 64];
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) partial[blockIdx.x] = sums[0] + sums[1] + (sums[2] + sums[3]);
}
template <typename G, bool STREAM>
__global__ __launch_bounds__(kThreads) void ds_adamw_squares_flat_kernel(const Flat *__restrict__ chunks, int64_t count, double *partial) {
  double sum = 0.0;
  for (int64_t c = (int64_t)blockIdx.x * kSquareChunks; c < count; c += (int64_t)gridDim.x * kSquareChunks) {
    const void *from[kSquareChunks];
    int left[kSquareChunks];
#pragma unroll
    for (int u = 0; u < kSquareChunks; ++u) {
      const Flat &f = chunks[c + u < count ? c + u : c];
      from[u] = global((const void *)f.grad), left[u] = c + u < count ? f.left : 0;
    }
    typename QuadOf<G>::Bits g[kSquareChunks][kEach];
#pragma unroll
    for (int u = 0; u < kSquareChunks; ++u)
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int j = (e * kThreads + threadIdx.x) * 4, more = left[u] - j;
        g[u][e] = ask_quad<G, STREAM>(from[u], j, more < 0 ? 0 : more < 4 ? more : 4);
      }
#pragma unroll
    for (int u = 0; u < kSquareChunks; ++u)
#pragma unroll
      for (int e = 0; e < kEach; ++e) add_squares<G>(g[u][e], sum);
  }
  put_sum(sum, partial);
}
template <typename G>
__global__ __launch_bounds__(kThreads) void ds_adamw_squares_rows_kernel(const Tensor *__restrict__ tensors, const Chunk *__restrict__ chunks, int64_t count, double *partial) {
  double sum = 0.0;
  for (int64_t c = blockIdx.x; c < count; c += gridDim.x) {
    const Chunk chunk = chunks[c];
    const Tensor &t = tensors[chunk.tensor];
    const Rows grad = rows_of(t.grad);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      int64_t i, j;
      int n;
      place_of(t, chunk.quad + e * kThreads + threadIdx.x, i, j, n);
      add_squares<G>(ask_quad<G, false>(grad.base, i * grad.stride + j, n), sum);
    }
  }
  put_sum(sum, partial);
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

int64_t square_groups(const Kind &k) {
  const int64_t chunks = k.end - k.begin;
  return std::min(k.flat ? (chunks + kSquareChunks - 1) / kSquareChunks : chunks, kSquareGroups);
}

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

// Is memory written twice, or read as a gradient and written?
bool written_twice(std::vector<Range> &ranges, const std::vector<Range> &grads) {
  std::sort(ranges.begin(), ranges.end(), [](const Range &a, const Range &b) { return a.begin < b.begin; });
  std::vector<Range> wholes;
  for (size_t k = 0; k < ranges.size(); ++k) {
    const Range &r = ranges[k];
    if (k && ranges[k - 1].begin == r.begin) return true;
    if (!r.whole) continue;
    if (!wholes.empty() && r.begin < wholes.back().end) return true;
    wholes.push_back(r);
  }
  for (const Range &g : grads) {
    if (!g.whole) continue;
    const auto behind = std::lower_bound(wholes.begin(), wholes.end(), g.end, [](const Range &w, uintptr_t end) { return w.begin < end; });
    if (behind != wholes.begin() && behind[-1].end > g.begin) return true;
  }
  return false;
}

}  // namespace

struct ds_adamw {
  int device = -1;
  void *memory = nullptr;
  const Tensor *tensors = nullptr;  // those of rows
  const Chunk *chunks = nullptr;    // theirs
  const Flat *flats = nullptr;      // those of tensors that are one row
  std::vector<Kind> kinds;
  int64_t elements = 0;
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
  std::vector<Range> written, grads;
  std::vector<std::pair<uint32_t, uint32_t>> order;  // kind and place in `tensors`
  for (size_t k = 0; k < n; ++k) {
    const ds_adamw_tensor &f = from[k];
    bool copied = false;
    DS_TRY(check_tensor(f, copied));
    const int64_t rows = f.param.rows, cols = f.param.cols;
    if (rows == 0 || cols == 0) continue;
    if (rows * cols > kMostElements - table.elements) return DS_ERANGE;
    table.elements += rows * cols;
    const bool eight = f.m.dtype == DS_MX8;
    const ds_matrix *all[] = {&f.param, &f.grad, &f.m, &f.v, copied ? &f.copy : nullptr};
    bool row = true;
    for (const ds_matrix *m : all) {
      if (!m) continue;
      row = row && one_row(*m, m->dtype >= DS_MX8);
      add_range(m == &f.grad ? grads : written, m->base, rows, cols, m->row_stride, m->dtype >= DS_MX8 ? 1 : ds_itemsize(m->dtype));
      if (m->dtype >= DS_MX8) add_range(written, m->scale, rows, ds_groups(cols), m->scale_stride, 1);
    }
    Tensor t{};
    t.param = ds_rows(&f.param), t.grad = ds_rows(&f.grad), t.m = ds_rows(&f.m), t.v = ds_rows(&f.v), t.copy = ds_rows(copied ? &f.copy : nullptr);
    t.rows = row ? 1 : rows, t.cols = row ? rows * cols : cols;
    t.quads = eight ? ds_groups(t.cols) * (kGroup / 4) : (t.cols + 3) / 4;
    t.number = (uint32_t)k, t.copy_dtype = copied ? f.copy.dtype : 0, t.decay = f.decay, t.rate = f.rate;
    order.emplace_back(f.param.dtype * 12 + f.grad.dtype * 4 + eight * 2 + row, (uint32_t)tensors.size());
    tensors.push_back(t);
  }
  if (written_twice(written, grads)) return DS_EOVERLAP;
  std::stable_sort(order.begin(), order.end(), [](const auto &a, const auto &b) { return a.first < b.first; });
  std::vector<Tensor> of_rows;
  std::vector<Chunk> chunks;
  std::vector<Flat> flats;
  for (size_t k = 0; k < order.size(); ++k) {
    const uint32_t kind = order[k].first;
    const Tensor &t = tensors[order[k].second];
    const bool flat = kind % 2;
    if (k == 0 || order[k - 1].first != kind)
      table.kinds.push_back({kind / 12, kind / 4 % 3, kind / 2 % 2, kind % 2, (int64_t)(flat ? flats.size() : chunks.size()), 0});
    if (flat) {
      const Kind &of = table.kinds.back();
      const int64_t m = of.eight ? 1 : 4, copy = ds_itemsize(t.copy_dtype);
      const auto at = [](const void *base, int64_t bytes) { return base ? (void *)((uint8_t *)base + bytes) : nullptr; };
      for (int64_t j = 0; j < t.cols; j += kQuads * 4)
        flats.push_back({at(t.param.base, j * ds_itemsize(of.param)), at(t.grad.base, j * ds_itemsize(of.grad)), at(t.m.base, j * m), at(t.v.base, j * m),
                         at(t.copy.base, j * copy), (uint8_t *)at(t.m.scale, j / kGroup), (uint8_t *)at(t.v.scale, j / kGroup),
                         (int32_t)std::min(t.cols - j, kQuads * 4), (uint32_t)j, t.number, t.copy_dtype, t.decay, t.rate});
    } else {
      for (int64_t quad = 0; quad < t.rows * t.quads; quad += kQuads) chunks.push_back({quad, (uint32_t)of_rows.size(), 0});
      of_rows.push_back(t);
    }
    table.kinds.back().end = (int64_t)(flat ? flats.size() : chunks.size());
  }
  DS_HIP_TRY(hipGetDevice(&table.device));
  if (tensors.empty()) return DS_OK;
  const size_t sizes[] = {of_rows.size() * sizeof(Tensor), chunks.size() * sizeof(Chunk), flats.size() * sizeof(Flat)};
  std::vector<uint8_t> all(sizes[0] + sizes[1] + sizes[2]);
  std::copy_n((const uint8_t *)of_rows.data(), sizes[0], all.data());
  std::copy_n((const uint8_t *)chunks.data(), sizes[1], all.data() + sizes[0]);
  std::copy_n((const uint8_t *)flats.data(), sizes[2], all.data() + sizes[0] + sizes[1]);
  const hipError_t e = hipMalloc(&table.memory, all.size());
  if (e == hipErrorOutOfMemory) {
    (void)hipGetLastError();
    return DS_ENOMEM;
  }
  DS_HIP_TRY(e);
  const uint8_t *at = (const uint8_t *)table.memory;
  table.tensors = (const Tensor *)at, table.chunks = (const Chunk *)(at + sizes[0]), table.flats = (const Flat *)(at + sizes[0] + sizes[1]);
  DS_HIP_TRY(hipMemcpy(table.memory, all.data(), all.size(), hipMemcpyHostToDevice));
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
      const auto launch = [&](auto kernel, auto... table_of) -> int {
        hipLaunchKernelGGL(kernel, dim3((uint32_t)groups), dim3(kThreads), 0, (hipStream_t)stream, table_of..., k.end - k.begin, partial);
        DS_HIP_TRY(hipGetLastError());
        return DS_OK;
      };
      if (!k.flat) return launch(ds_adamw_squares_rows_kernel<G>, table->tensors, table->chunks + k.begin);
      return table->elements < kStream ? launch(ds_adamw_squares_flat_kernel<G, false>, table->flats + k.begin)
                                       : launch(ds_adamw_squares_flat_kernel<G, true>, table->flats + k.begin);
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
  const auto amount = [](double x) { return x >= 0.0 && x <= (double)FLT_MAX; };
  // (the reciprocal takes no subnormal numbers, which eps alone is where v is 0)
  if (!amount(f.rate) || !amount(f.eps) || (f.eps > 0.0 && f.eps < (double)FLT_MIN) || !share(f.beta1) || !share(f.beta2) || !std::isfinite(f.grad_scale) || !(f.most_norm >= 0.0) || !f.step ||
      ds_misaligned(f.step, 8) || ds_misaligned(f.rate_now, 4) || ds_misaligned(f.squares, 8) || (f.most_norm > 0.0 && !f.squares))
    return DS_EINVAL;
  DS_TRY(on_its_device(table));
  const Settings s{f.rate, std::log(f.beta1), std::log(f.beta2), f.grad_scale, f.most_norm, f.step, f.rate_now, f.squares, (float)f.beta1,
                   (float)f.beta2, (float)(1.0 - f.beta1), (float)(1.0 - f.beta2), (float)f.eps, mix((uint32_t)f.seed ^ mix((uint32_t)(f.seed >> 32)))};
  for (const Kind &k : table->kinds) {
    const int64_t count = k.end - k.begin;
    DS_TRY(ds_with_type(k.param, [&](auto type) -> int {
      typedef decltype(type) P;
      return ds_with_type(k.grad, [&](auto grad) -> int {
        typedef decltype(grad) G;
        const auto launch = [&](auto kernel, auto... table_of) -> int {
          hipLaunchKernelGGL(kernel, dim3((uint32_t)std::min(count, kMaxGrid)), dim3(kThreads), 0, (hipStream_t)stream, table_of..., count, s);
          DS_HIP_TRY(hipGetLastError());
          return DS_OK;
        };
        if (!k.flat)
          return k.eight ? launch(ds_adamw_rows_kernel<P, G, true>, table->tensors, table->chunks + k.begin)
                         : launch(ds_adamw_rows_kernel<P, G, false>, table->tensors, table->chunks + k.begin);
        const Flat *flats = table->flats + k.begin;
        if (table->elements < kStream)
          return k.eight ? launch(ds_adamw_flat_kernel<P, G, true, false>, flats) : launch(ds_adamw_flat_kernel<P, G, false, false>, flats);
        return k.eight ? launch(ds_adamw_flat_kernel<P, G, true, true>, flats) : launch(ds_adamw_flat_kernel<P, G, false, true>, flats);
      });
    }));
  }
  return DS_OK;
}
