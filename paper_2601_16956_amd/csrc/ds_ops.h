// What the operators of the training step share: the checks of their arguments, the element types, the codes of
// checkpoints in 8 bits, the activations, and sums over a wavefront.  Not part of the ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

#include "ds_internal.h"

// ---- host: the checks ---------------------------------------------------------------------------------------

constexpr int64_t kMaxExtent = 0x7fffffff;  // rows, columns: kernels count them in 32 bits
constexpr int64_t kMaxGrid = 1 << 22;       // work-groups of a launch, whose threads are fewer than 2^32
constexpr int kGroup = 32;                  // columns that share a scale in a checkpoint in 8 bits

inline bool ds_is_float(uint32_t dtype) { return dtype == DS_F32 || dtype == DS_BF16 || dtype == DS_F16; }
inline bool ds_is_half(uint32_t dtype) { return dtype == DS_BF16 || dtype == DS_F16; }
inline int64_t ds_groups(int64_t cols) { return (cols + kGroup - 1) / kGroup; }

// Is `m` a matrix (of ROWS, if `rows_only`)?  Strides of extents of 0 and 1 mean nothing and are not looked at.
inline int ds_check_matrix(const ds_matrix *m, bool rows_only) {
  if (!m || m->reserved || m->rows < 0 || m->cols < 0) return DS_EINVAL;
  const bool mx8 = m->dtype == DS_MX8;
  if (!mx8 && !ds_is_float(m->dtype)) return DS_EINVAL;
  if (m->rows > kMaxExtent || m->cols > kMaxExtent) return DS_ERANGE;
  if (!mx8 && (m->scale || m->scale_stride)) return DS_EINVAL;
  if (m->rows == 0 || m->cols == 0) return DS_OK;
  const uint64_t size = mx8 ? 1 : (uint64_t)ds_itemsize(m->dtype);
  if (!m->base || ((uintptr_t)m->base & (size - 1))) return DS_EINVAL;
  const bool r = m->rows > 1, c = m->cols > 1;
  if ((r && m->row_stride < 1) || (c && m->col_stride < 1)) return DS_EINVAL;
  const bool in_rows = (!c || m->col_stride == 1) && (!r || m->row_stride >= m->cols);
  const bool in_cols = (!r || m->row_stride == 1) && (!c || m->col_stride >= m->rows);
  if (!in_rows && (!in_cols || rows_only || mx8)) return DS_EINVAL;
  // the last element's distance from the first fits 63 bits
  const __int128 last = (__int128)(r ? m->row_stride : 0) * (m->rows - 1) + (__int128)(c ? m->col_stride : 0) * (m->cols - 1);
  if (last * (__int128)size > (__int128)INT64_MAX) return DS_ERANGE;
  if (mx8) {
    if (!m->scale || (r && m->scale_stride < ds_groups(m->cols))) return DS_EINVAL;
    if (r && (__int128)m->scale_stride * (m->rows - 1) > (__int128)INT64_MAX) return DS_ERANGE;
  }
  return DS_OK;
}

inline bool ds_same_extents(const ds_matrix *a, const ds_matrix *b) { return a->rows == b->rows && a->cols == b->cols; }
inline bool ds_misaligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

#define DS_TRY(expr)              \
  do {                            \
    const int _rc = (expr);       \
    if (_rc != DS_OK) return _rc; \
  } while (0)

// Calls f with a value of the element type that `dtype` names.
template <typename F>
inline int ds_with_type(uint32_t dtype, F f) {
  if (dtype == DS_F32) return f(float());
  if (dtype == DS_BF16) return f(__hip_bfloat16());
  return f(__half());
}

// ---- device: elements ----------------------------------------------------------------------------------------

// Rows start wherever their strides put them, and gfx950 runs with unaligned global access: eight neighbouring elements
// are one vector access (two of floats) at any address that is a multiple of the element.
typedef uint32_t ds_u32x2 __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t ds_u32x4 __attribute__((ext_vector_type(4), aligned(1)));

typedef float ds_f32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 ds_bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 ds_f16x8 __attribute__((ext_vector_type(8)));

// Eight elements as 32-bit floats.
struct Eight {
  float v[8];
};

__device__ inline float bf16_to_float(uint32_t bits) { return __uint_as_float(bits << 16); }
// to nearest, ties to even; a NaN stays one
__device__ inline uint32_t float_to_bf16(float x) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x);
}
__device__ inline uint32_t float_to_f16(float x) { return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x); }
__device__ inline float f16_to_float(uint32_t bits) { return (float)__builtin_bit_cast(_Float16, (uint16_t)bits); }

template <typename T>
struct Elem;
template <>
struct Elem<float> {
  static __device__ inline float get(const void *p, int64_t i) { return ((const float *)p)[i]; }
  static __device__ inline void put(void *p, int64_t i, float x) { ((float *)p)[i] = x; }
  static __device__ inline Eight get8(const void *p, int64_t i) {
    const ds_u32x4 *q = (const ds_u32x4 *)((const float *)p + i);
    const ds_u32x4 a = q[0], b = q[1];
    Eight e;
#pragma unroll
    for (int k = 0; k < 4; ++k) e.v[k] = __uint_as_float(a[k]), e.v[4 + k] = __uint_as_float(b[k]);
    return e;
  }
  static __device__ inline void put8(void *p, int64_t i, const Eight &e) {
    ds_u32x4 a, b;
#pragma unroll
    for (int k = 0; k < 4; ++k) a[k] = __float_as_uint(e.v[k]), b[k] = __float_as_uint(e.v[4 + k]);
    ds_u32x4 *q = (ds_u32x4 *)((float *)p + i);
    q[0] = a, q[1] = b;
  }
};
template <>
struct Elem<__hip_bfloat16> {
  static __device__ inline float get(const void *p, int64_t i) { return bf16_to_float(((const uint16_t *)p)[i]); }
  static __device__ inline void put(void *p, int64_t i, float x) { ((uint16_t *)p)[i] = (uint16_t)float_to_bf16(x); }
  static __device__ inline Eight get8(const void *p, int64_t i) {
    const ds_u32x4 a = *(const ds_u32x4 *)((const uint16_t *)p + i);
    Eight e;
#pragma unroll
    for (int k = 0; k < 4; ++k) e.v[2 * k] = __uint_as_float(a[k] << 16), e.v[2 * k + 1] = __uint_as_float(a[k] & 0xffff0000u);
    return e;
  }
  static __device__ inline void put8(void *p, int64_t i, const Eight &e) {
    *(ds_u32x4 *)((uint16_t *)p + i) = __builtin_bit_cast(ds_u32x4, __builtin_convertvector(__builtin_bit_cast(ds_f32x8, e), ds_bf16x8));
  }
};
template <>
struct Elem<__half> {
  static __device__ inline float get(const void *p, int64_t i) { return f16_to_float(((const uint16_t *)p)[i]); }
  static __device__ inline void put(void *p, int64_t i, float x) { ((uint16_t *)p)[i] = (uint16_t)float_to_f16(x); }
  static __device__ inline Eight get8(const void *p, int64_t i) {
    const ds_u32x4 a = *(const ds_u32x4 *)((const uint16_t *)p + i);
    Eight e;
#pragma unroll
    for (int k = 0; k < 4; ++k) e.v[2 * k] = f16_to_float(a[k] & 0xffffu), e.v[2 * k + 1] = f16_to_float(a[k] >> 16);
    return e;
  }
  static __device__ inline void put8(void *p, int64_t i, const Eight &e) {
    *(ds_u32x4 *)((uint16_t *)p + i) = __builtin_bit_cast(ds_u32x4, __builtin_convertvector(__builtin_bit_cast(ds_f32x8, e), ds_f16x8));
  }
};

// Eight elements of a vector whose type is known at run time only (a bias, gamma: few of them, read once a row or tile).
__device__ inline Eight get8_any(const void *p, uint32_t dtype, int64_t i) {
  return dtype == DS_F32 ? Elem<float>::get8(p, i) : dtype == DS_BF16 ? Elem<__hip_bfloat16>::get8(p, i) : Elem<__half>::get8(p, i);
}

// The first n <= 8 of the eight from i on (n <= 0: none of them); the others are 0 and are not read, or not written.
template <typename T>
__device__ inline Eight get_up_to8(const void *p, int64_t i, int n) {
  if (n >= 8) return Elem<T>::get8(p, i);
  Eight e;
#pragma unroll
  for (int k = 0; k < 8; ++k) e.v[k] = k < n ? Elem<T>::get(p, i + k) : 0.f;
  return e;
}
template <typename T>
__device__ inline void put_up_to8(void *p, int64_t i, int n, const Eight &e) {
  if (n >= 8) return Elem<T>::put8(p, i, e);
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (k < n) Elem<T>::put(p, i + k, e.v[k]);
}
// In two halves: the bits of several such vectors are on their way together, where making floats of one would wait for it.
struct AnyBits {
  ds_u32x4 w[2];
};
__device__ inline AnyBits ask_up_to8_any(const void *p, uint32_t dtype, int64_t i, int n) {
  AnyBits b = {};
  if (!p || n <= 0) return b;
  if (dtype == DS_F32) {
    const uint32_t *q = (const uint32_t *)p + i;
    if (n >= 8) b.w[0] = *(const ds_u32x4 *)q, b.w[1] = *(const ds_u32x4 *)(q + 4);
    else
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < n) b.w[k / 4][k % 4] = q[k];
  } else {
    const uint16_t *q = (const uint16_t *)p + i;
    if (n >= 8) b.w[0] = *(const ds_u32x4 *)q;
    else
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < n) b.w[0][k / 2] |= (uint32_t)q[k] << (16 * (k % 2));
  }
  return b;
}
// `without`: what stands for a vector that there is none of.
__device__ inline Eight value_any(const AnyBits &b, const void *p, uint32_t dtype, float without) {
  Eight e;
  if (!p) {
#pragma unroll
    for (int k = 0; k < 8; ++k) e.v[k] = without;
    return e;
  }
  return get8_any(&b, dtype, 0);
}
__device__ inline Eight get_up_to8_any(const void *p, uint32_t dtype, int64_t i, int n, float without) {
  return value_any(ask_up_to8_any(p, dtype, i, n), p, dtype, without);
}

// ---- device: checkpoints in 8 bits -----------------------------------------------------------------------------

// A lane holds eight neighbouring columns, from a multiple of 8 on; four lanes from a multiple of 4 on hold a group of 32.
// What a lane knows of the group is the largest magnitude, as bits: among floats without their sign the order of the
// bits is that of the values, with infinities and NaN above all.
__device__ inline uint32_t magnitude8(const Eight &e) {
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const uint32_t m = __float_as_uint(e.v[k]) & 0x7fffffffu;
    top = m > top ? m : top;
  }
  return top;
}
// The largest of four neighbouring lanes' (quad_perm 1,0,3,2, then 2,3,0,1).
__device__ inline uint32_t max_of_four_lanes(uint32_t m) {
  uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xf, 0xf, true);
  m = o > m ? o : m;
  o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xf, 0xf, true);
  return o > m ? o : m;
}
// The scale byte of a group whose largest magnitude has these bits.
__device__ inline uint32_t mx8_scale(uint32_t top) {
  return top == 0 ? 0u : top >= 0x7f800000u ? 255u : (top >> 23) > 1u ? top >> 23 : 1u;
}
// Eight codes under that scale, as bytes.  x * 2^(133 - scale) is at most 128 steps; added to 1.5 * 2^23 in one operation, whose
// rounding, to even, is the only one, it leaves the whole number of steps in the low bits.
__device__ inline ds_u32x2 mx8_codes(const Eight &e, uint32_t scale) {
  constexpr float kWhole = 12582912.f;
  uint32_t q[8];
  if (scale < 6u) {  // the factor is no float: magnitudes below 2^-121
#pragma unroll
    for (int k = 0; k < 8; ++k) q[k] = (uint32_t)(int)__builtin_amdgcn_fmed3f(__builtin_rintf(ldexpf(e.v[k], 133 - (int)scale)), -127.f, 127.f);
  } else {
    const float steps = __uint_as_float((260u - (scale == 255u ? 133u : scale)) << 23);  // 2^(133 - scale)
#pragma unroll
    for (int k = 0; k < 8; ++k)
      q[k] = __float_as_uint(__builtin_amdgcn_fmed3f(__builtin_fmaf(e.v[k], steps, kWhole), kWhole - 127.f, kWhole + 127.f));
  }
  ds_u32x2 r;
#pragma unroll
  for (int h = 0; h < 2; ++h) {  // the low bytes of four words: two, two, then all
    const uint32_t low = __builtin_amdgcn_perm(q[4 * h + 1], q[4 * h], 0x0c0c0400u), high = __builtin_amdgcn_perm(q[4 * h + 3], q[4 * h + 2], 0x04000c0cu);
    r[h] = scale == 255u ? 0u : low | high;
  }
  return r;
}
// The step of a group, 2^(scale - 133); NaN where the group has no values.
__device__ inline float mx8_step(uint32_t scale) {
  return scale == 255u ? __uint_as_float(0x7fc00000u) : ldexpf(1.f, (int)scale - 133);
}
__device__ inline Eight mx8_values(ds_u32x2 codes, float step) {
  Eight e;
#pragma unroll
  for (int k = 0; k < 8; ++k) e.v[k] = (float)((int)(codes[k / 4] << (24 - 8 * (k % 4))) >> 24) * step;
  return e;
}

// A matrix in rows as kernels have it.  scale is for checkpoints only.
struct Rows {
  void *base;
  int64_t stride;  // elements
  uint8_t *scale;
  int64_t scale_stride;
};
inline Rows ds_rows(const ds_matrix *m) {
  if (!m) return Rows{nullptr, 0, nullptr, 0};
  return Rows{m->base, m->rows > 1 ? m->row_stride : 0, m->scale, m->rows > 1 ? m->scale_stride : 0};
}

// Marks the type of a checkpoint in 8 bits where a template takes an element type.
struct Mx8 {};

// The first n <= 8 of eight values from column j (a multiple of 8) of row i on; the others are 0.  In two halves, so that a kernel can
// ask for a row long before it computes on it: ask() loads the bits, value() makes floats of them.
template <typename T>
struct RowsOf {
  struct Bits {
    ds_u32x4 w[sizeof(T) / 2];
  };
  static __device__ inline Bits ask(const Rows &m, int64_t i, int64_t j, int n) {
    Bits b = {};
    const T *from = (const T *)m.base + i * m.stride + j;
    if (n >= 8) {
#pragma unroll
      for (int k = 0; k < (int)sizeof(T) / 2; ++k) b.w[k] = ((const ds_u32x4 *)from)[k];
    } else if (sizeof(T) == 4) {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < n) b.w[k / 4][k % 4] = ((const uint32_t *)from)[k];
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < n) b.w[0][k / 2] |= (uint32_t)((const uint16_t *)from)[k] << (16 * (k % 2));
    }
    return b;
  }
  static __device__ inline Eight value(const Bits &b, int) { return Elem<T>::get8(&b, 0); }
  static __device__ inline Eight get(const Rows &m, int64_t i, int64_t j, int n) { return value(ask(m, i, j, n), n); }
};
template <>
struct RowsOf<Mx8> {
  struct Bits {
    ds_u32x2 codes;
    uint32_t scale;
  };
  static __device__ inline Bits ask(const Rows &m, int64_t i, int64_t j, int n) {
    Bits b = {};
    const uint8_t *codes = (const uint8_t *)m.base + i * m.stride + j;
    if (n > 0) b.scale = m.scale[i * m.scale_stride + j / kGroup];
    if (n >= 8) b.codes = *(const ds_u32x2 *)codes;
    else
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < n) b.codes[k / 4] |= (uint32_t)codes[k] << (8 * (k % 4));
    return b;
  }
  static __device__ inline Eight value(const Bits &b, int n) {
    Eight e = mx8_values(b.codes, mx8_step(b.scale));
    if (n < 8) {  // a step of NaN is not to reach the places beyond the row
#pragma unroll
      for (int k = 0; k < 8; ++k) e.v[k] = k < n ? e.v[k] : 0.f;
    }
    return e;
  }
  static __device__ inline Eight get(const Rows &m, int64_t i, int64_t j, int n) { return value(ask(m, i, j, n), n); }
};

// Leaves eight values (n <= 8 of them in the row, the others 0) of row i from column j on in a checkpoint.  All lanes of
// the wavefront take part; four neighbouring ones hold a group.
__device__ inline void mx8_put(const Rows &m, int64_t i, int64_t j, int n, const Eight &e) {
  const uint32_t scale = mx8_scale(max_of_four_lanes(magnitude8(e)));
  const ds_u32x2 q = mx8_codes(e, scale);
  if (n <= 0) return;
  uint8_t *codes = (uint8_t *)m.base + i * m.stride + j;
  if (n >= 8) *(ds_u32x2 *)codes = q;
  else
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < n) codes[k] = (uint8_t)(q[k / 4] >> (8 * (k % 4)));
  if (j % kGroup == 0) m.scale[i * m.scale_stride + j / kGroup] = (uint8_t)scale;
}

// ---- device: activations ---------------------------------------------------------------------------------------

// FULL: for results of 32 bits, every factor to a few units of the last place, out to where results are subnormal.  Else, for results
// that are rounded to 16 bits, the exponential is v_exp_f32 of a rounded product, off by up to |argument| * 2^-24 of itself (4e-6 at
// -80), and the reciprocal v_rcp_f32, off by one unit: far below the rounding that follows.  (What FULL costs, f32: the backward
// pass of 8192 x 3584 0 to 1 %, a product 8192 x 1024 x 8192 with GELU 195 and 197 us, with its tanh form 177 and 184.)

// 1 / x for 1 <= x <= 8, to a unit of the last place: a step of Newton's behind the approximation.
__device__ inline float reciprocal(float x) {
  const float r = __builtin_amdgcn_rcpf(x);
  return __builtin_fmaf(__builtin_fmaf(-x, r, 1.f), r, r);
}
// p = 1 / (1 + exp(-x)), and q = 1 - p without the cancellation.
template <bool FULL>
__device__ inline float sigmoid(float x, float &q) {
  if (FULL) {  // exp of what is not positive cannot overflow
    const float e = expf(-__builtin_fabsf(x)), high = reciprocal(1.f + e), low = e * high;
    q = x < 0.f ? high : low;
    return x < 0.f ? low : high;
  }
  // exp overflows to infinity for very negative x, and the reciprocal is then 0, its limit (below 2^-126 so too)
  const float p = __builtin_amdgcn_rcpf(1.f + __expf(-x));
  q = 1.f - p;
  return p;
}
// The part of the normal distribution below z, and gauss = exp(-z^2 / 2).  Below -w it is gauss * t P(t), t = 1 / (1 + 0.35 w), P the
// polynomial of eight degrees whose largest error of itself over 0 <= w <= 20 is least: 4.4e-8 (a weighted least-squares
// fit to exp(w^2 / 2) erfc(w / sqrt(2)) / 2).  In units of itself: 1 + erf loses its digits where z is negative, all of
// them from -5.5 on.  Beyond 20 nothing is left in 32 bits.
template <bool FULL>
__device__ inline float normal_below(float z, float &gauss) {
  const float far = __builtin_fabsf(z), w = far > 20.f ? 20.f : far, square = w * w;
  if (FULL) {
    gauss = expf(-0.5f * square);
    gauss = __builtin_fmaf(-0.5f * __builtin_fmaf(w, w, -square), gauss, gauss);  // what the square's rounding left out
  } else {
    gauss = __expf(-0.5f * square);
  }
  const float t = FULL ? reciprocal(__builtin_fmaf(0.35f, w, 1.f)) : __builtin_amdgcn_rcpf(__builtin_fmaf(0.35f, w, 1.f));
  constexpr float P[9] = {0.139622584f, 0.139836043f, 0.120061718f, 0.104427479f, -0.0201176777f, 0.154166251f, -0.250737578f, 0.141272306f, -0.0285311043f};
  float sum = P[8];
#pragma unroll
  for (int k = 7; k >= 0; --k) sum = __builtin_fmaf(sum, t, P[k]);
  const float tail = gauss * (sum * t);
  return z < 0.f ? tail : 1.f - tail;
}
constexpr float kGeluTanh = 0.7978845608028654f;  // sqrt(2 / pi)
constexpr float kGeluCube = 0.044715f;

// (1 + tanh(u)) / 2 = 1 / (1 + exp(-2 u)), so the tanh form is z * sigmoid(2 u).  At z = -infinity the products would be
// infinity times 0; the limit is 0.
template <uint32_t ACT, bool FULL>
__device__ inline float activation(float z) {
  float other;
  if (ACT == DS_ACT_GELU) return z == -__builtin_inff() ? 0.f : z * normal_below<FULL>(z, other);
  if (ACT == DS_ACT_GELU_TANH) return z == -__builtin_inff() ? 0.f : z * sigmoid<FULL>(2.f * kGeluTanh * (z + kGeluCube * z * z * z), other);
  if (ACT == DS_ACT_SILU) return z == -__builtin_inff() ? 0.f : z * sigmoid<FULL>(z, other);
  return z;
}
// (Where gauss or p q is 0, z may be infinite.)
template <uint32_t ACT, bool FULL>
__device__ inline float activation_slope(float z) {
  if (ACT == DS_ACT_GELU) {
    float gauss;
    const float p = normal_below<FULL>(z, gauss);
    return p + (gauss == 0.f ? 0.f : z * gauss * 0.3989422804014327f);
  }
  if (ACT == DS_ACT_GELU_TANH) {
    float q;
    const float p = sigmoid<FULL>(2.f * kGeluTanh * (z + kGeluCube * z * z * z), q), flat = p * q;
    return p + (flat == 0.f ? 0.f : z * flat * 2.f * kGeluTanh * (1.f + 3.f * kGeluCube * z * z));
  }
  if (ACT == DS_ACT_SILU) {
    float q;
    const float p = sigmoid<FULL>(z, q), flat = p * q;
    return p + (flat == 0.f ? 0.f : z * flat);
  }
  return 1.f;
}

template <typename F>
inline int ds_with_act(uint32_t act, F f) {
  if (act == DS_ACT_GELU) return f(std::integral_constant<uint32_t, DS_ACT_GELU>());
  if (act == DS_ACT_GELU_TANH) return f(std::integral_constant<uint32_t, DS_ACT_GELU_TANH>());
  if (act == DS_ACT_SILU) return f(std::integral_constant<uint32_t, DS_ACT_SILU>());
  return f(std::integral_constant<uint32_t, DS_ACT_NONE>());
}

// ---- device: sums ------------------------------------------------------------------------------------------------

// The sum over the wavefront, in every lane.
__device__ inline float wave_sum(float x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d, 64);
  return x;
}

// out0[j] = partial[0][j] + partial[1][j] + ... over `parts` lines of `cols`, in an order that only their number decides; out1
// likewise from the lines behind those.  Either may be NULL.
int ds_launch_sum_parts(const float *partial, int64_t parts, int64_t cols, float *out0, float *out1, hipStream_t stream);
