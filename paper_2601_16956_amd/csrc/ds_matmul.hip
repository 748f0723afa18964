// c = act(a b + bias) + residual on the matrix cores.
//
// Three ways, by the sizes (choose()):
//   tiles     a work-group has a tile of 64 x 64 to 256 x 256 of c and walks along k; the operands go from memory to LDS without
//             passing registers, in either order of each; few tiles are split along k, and joined by a second launch.
//             Operands that are no whole 16-byte pieces, or checkpoints in 8 bits, are laid out in the workspace first.  Bound by
//             the matrix cores and, at the largest sizes, by the power that they draw: 16384 x 3584 x 8192 in bfloat16
//             about 720 us, 1.34 PFLOP/s, with a residual 770 (a library's product 626 to 728 us, as data and card let it);
//             8192^3 about 790 us (690 to 796).  Zeros instead of normal numbers run a fifth faster.
//   few rows  at most 16 rows on a weight [out, in], save where n is small and k long: bound by reading
//             the weight, 1 x 8192 x 3584 in 15 us, 3.9 TB/s.
//   simple    whatever is left: products of less than 2^18 multiplications, and lines beyond 2^21 elements.
//
// Always: 32-bit sums; v_mfma_f32_16x16x32 with the operands exchanged, so that a lane's four results are neighbouring
// columns of one row; the sums go through LDS once more, to leave a lane eight neighbouring columns for the epilogue: the
// bias, the checkpoint of z (four lanes hold a group of 32), the activation, the residual and the one rounding.

#include <type_traits>

#include "ds_choice.h"
#include "ds_ops.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
static_assert(kMaxTiles <= kMaxGrid && kMaxTiles * 512 < (int64_t)1 << 32, "a launch's threads");

struct Epilogue {
  Rows c, residual, saved;
  const void *bias;
  int64_t m, n;
  uint32_t c_dtype, bias_dtype, act;
};

__device__ inline f32x4 mfma(u32x4 x, u32x4 y, f32x4 sum, __hip_bfloat16) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), sum, 0, 0, 0);
}
__device__ inline f32x4 mfma(u32x4 x, u32x4 y, f32x4 sum, __half) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), sum, 0, 0, 0);
}

template <uint32_t ACT, bool FULL>
__device__ inline void activate8(Eight &z) {
#pragma unroll
  for (int k = 0; k < 8; ++k) z.v[k] = activation<ACT, FULL>(z.v[k]);
}

// The first n <= 8 of eight biases from column j on, zeros where there is none.
__device__ inline Eight bias8(const Epilogue &e, int64_t j, int n) { return get_up_to8_any(e.bias, e.bias_dtype, j, n, 0.f); }

// Eight sums of row i from column j (a multiple of 8) on, n <= 8 of them in c, leave by the epilogue; T: c's type.  All lanes of the
// wavefront take part, four neighbouring ones with a group of 32 columns.  The residual's bits have been asked for before.
template <typename T>
__device__ inline void finish8(const Epilogue &e, int64_t i, int64_t j, int n, Eight z, const Eight &bias, const typename RowsOf<T>::Bits &residual) {
#pragma unroll
  for (int k = 0; k < 8; ++k) z.v[k] += bias.v[k];
  if (e.saved.base) {
    Eight s = z;
    if (n < 8) {
#pragma unroll
      for (int k = 0; k < 8; ++k) s.v[k] = k < n ? z.v[k] : 0.f;
    }
    mx8_put(e.saved, i, j, n, s);
  }
  if (e.act == DS_ACT_GELU) activate8<DS_ACT_GELU, sizeof(T) == 4>(z);
  else if (e.act == DS_ACT_GELU_TANH) activate8<DS_ACT_GELU_TANH, sizeof(T) == 4>(z);
  else if (e.act == DS_ACT_SILU) activate8<DS_ACT_SILU, sizeof(T) == 4>(z);
  if (n <= 0) return;
  if (e.residual.base) {
    const Eight r = RowsOf<T>::value(residual, 8);
#pragma unroll
    for (int k = 0; k < 8; ++k) z.v[k] += r.v[k];
  }
  put_up_to8<T>(e.c.base, i * e.c.stride + j, n, z);
}
template <typename T>
__device__ inline typename RowsOf<T>::Bits residual8(const Epilogue &e, int64_t i, int64_t j, int n) {
  typename RowsOf<T>::Bits r = {};
  if (e.residual.base) r = RowsOf<T>::ask(e.residual, i, j, n);
  return r;
}
template <typename F>
__device__ inline void with_c_type(const Epilogue &e, F f) {
  if (e.c_dtype == DS_F32) f(float());
  else if (e.c_dtype == DS_BF16) f(__hip_bfloat16());
  else f(__half());
}
__device__ inline int columns_of(const Epilogue &e, int64_t i, int64_t j) {
  const int64_t left = i < e.m ? e.n - j : 0;
  return (int)(left < 0 ? 0 : left < 8 ? left : 8);
}

// ---- any operands ------------------------------------------------------------------------------------------------------

// A work-group of four wavefronts has a tile of 64 x 64 and walks along k in steps of 32.  Each thread brings eight neighbouring elements
// of either operand through registers into LDS, the next step's while the matrix instructions run on this one's; both
// operands lie in LDS with k last.  A wavefront has 16 rows of the tile.  (390 TFLOP/s at 16384 x 3584 x 8192.)
constexpr int kTile = 64, kDeep = 32, kPitch = kDeep + 8;

// Eight neighbouring elements of an operand for the LDS: of one p from k on (k_last), or of one k from p on.  Those beyond
// the matrix are 0.
template <typename T>
__device__ inline u32x4 bring8(const Operand &o, int64_t p, int64_t k, int64_t depth) {
  const int64_t line = o.k_last ? p : k, at = o.k_last ? k : p;
  const int64_t lines = o.k_last ? o.extent : depth, length = o.k_last ? depth : o.extent;
  const int64_t left = line < lines ? length - at : 0;
  const int n = (int)(left < 0 ? 0 : left < 8 ? left : 8);
  if (o.scale) {
    const Rows rows{const_cast<void *>(o.base), o.ld, const_cast<uint8_t *>(o.scale), o.scale_stride};
    const Eight e = RowsOf<Mx8>::get(rows, line, at, n);
    u32x4 r;
    Elem<T>::put8(&r, 0, e);
    return r;
  }
  u32x4 r = {0, 0, 0, 0};
  const uint16_t *q = (const uint16_t *)o.base + line * o.ld + at;
  if (n >= 8) return *(const ds_u32x4 *)q;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) r[i / 2] |= (uint32_t)q[i] << (16 * (i % 2));
  return r;
}

// bring8's place in the tile for this thread, and where it goes in LDS ([kTile][kPitch]).
__device__ inline void place(bool k_last, int &p, int &k) {
  const int t = threadIdx.x;
  if (k_last) p = t / 4, k = t % 4 * 8;
  else p = t % 8 * 8, k = t / 8;
}
__device__ inline void put_in_lds(uint16_t *lds, bool k_last, u32x4 x) {
  int p, k;
  place(k_last, p, k);
  if (k_last) {
    *(u32x4 *)(lds + p * kPitch + k) = x;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) lds[(p + i) * kPitch + k] = (uint16_t)(x[i / 2] >> (16 * (i % 2)));
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void ds_matmul_kernel(Operand a, Operand b, Epilogue e, int64_t depth, uint32_t across) {
  __shared__ union {
    struct {
      alignas(16) uint16_t a[kTile * kPitch], b[kTile * kPitch];
    } in;
    float out[kTile][kTile + 4];
  } lds;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t p0 = (int64_t)(blockIdx.x / across) * kTile, q0 = (int64_t)(blockIdx.x % across) * kTile;
  int pa, ka, pb, kb;
  place(a.k_last, pa, ka);
  place(b.k_last, pb, kb);
  f32x4 sum[4] = {};
  u32x4 na = {}, nb = {};
  if (depth > 0) na = bring8<T>(a, p0 + pa, ka, depth), nb = bring8<T>(b, q0 + pb, kb, depth);
  for (int64_t k = 0; k < depth; k += kDeep) {
    put_in_lds(lds.in.a, a.k_last, na);
    put_in_lds(lds.in.b, b.k_last, nb);
    __syncthreads();
    if (k + kDeep < depth) na = bring8<T>(a, p0 + pa, k + kDeep + ka, depth), nb = bring8<T>(b, q0 + pb, k + kDeep + kb, depth);
    const u32x4 x = *(const u32x4 *)(lds.in.a + (wave * 16 + lane % 16) * kPitch + lane / 16 * 8);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const u32x4 y = *(const u32x4 *)(lds.in.b + (t * 16 + lane % 16) * kPitch + lane / 16 * 8);
      sum[t] = mfma(y, x, sum[t], T());
    }
    __syncthreads();
  }
#pragma unroll
  for (int t = 0; t < 4; ++t) *(f32x4 *)&lds.out[wave * 16 + lane % 16][t * 16 + lane / 16 * 4] = sum[t];
  __syncthreads();
  with_c_type(e, [&](auto type) {
    typedef decltype(type) C;
    for (int r = 0; r < 2; ++r) {
      const int row = r * 32 + threadIdx.x / 8, col = threadIdx.x % 8 * 8;
      const int64_t i = p0 + row, j = q0 + col;
      const int n = columns_of(e, i, j);
      Eight z;
#pragma unroll
      for (int k = 0; k < 8; ++k) z.v[k] = lds.out[row][col + k];
      finish8<C>(e, i, j, n, z, bias8(e, j, n), residual8<C>(e, i, j, n));
    }
  });
}

// ---- tiles whose operands go to LDS directly ---------------------------------------------------------------------

// An operand as these kernels have it: 16-byte aligned, every line a whole number of 16-byte pieces apart and long.
struct Source {
  const uint8_t *base;
  int64_t ld;      // bytes
  int64_t extent;  // of p
};

struct TileArgs {
  Source a, b;
  int64_t depth;
  uint32_t tiles_m, tiles_n, splits;
  float *partial;  // [splits][m][n], or NULL: the epilogue follows at once
};

// Lane l of a wavefront brings 16 bytes from resource + offset to LDS at m0 + 16 l.  An offset of kNowhere reads zeros.
// Written by hand because the compiler would otherwise wait for the transfers of the next stage before it reads this one.  It does not
// look into the assembly for hazards either: a load may read a scalar register that a vector instruction has written (the resource's,
// by v_readfirstlane) five wait states later at the earliest, and m0 one.  (They cost nothing that can be measured.)
// m0 is an operand, so that the compiler writes it: it takes m0 to keep what it wrote there, and heeds no clobber of it.
constexpr uint32_t kNowhere = 0x80000000u;
__device__ inline void to_lds(uint32_t lds, uint32_t offset, u32x4 resource) {
  asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(lds), "v"(offset), "s"(resource) : "memory");
}
// All but the last LATER transfers of this wavefront are done, and what it has read of LDS is in registers; then the same
// holds for the work-group.
template <int LATER>
__device__ inline void stage_is_there() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LATER) : "memory");
}

// The part of one operand that a work-group stages: P lines or columns, kStep of k.
//   K_LAST: LDS holds P rows of 128 bytes, eight pieces of eight k; piece c of row r is at c ^ (r % 8).  A read takes 16 lanes
//     at a time, lanes 0-3, 12-15 and 20-27 first: rows 0-3 and 12-15 at one c and rows 4-11 at the next, which then lie in
//     different banks.  (Rows of 64 bytes, so that a stage is half as deep, make twice the requests of the L2: 8192^3
//     took a tenth longer so, 958 us against 876 in the loop of the time.)
//   else: LDS holds kStep rows of P elements.  A lane's eight k are then in eight rows: ds_read_b64_tr_b16 reads four rows of 16
//     elements with 16 lanes and gives each lane one column of them.  Pairs of pieces are exchanged by the row, so that
//     the 32 lanes of a pass, eight rows of 32 bytes, meet every bank once.
template <int P, int WAVES, bool K_LAST>
struct Stage {
  static constexpr int kBytes = P * kStep * 2, kLoads = kBytes / 1024 / WAVES, kLine = P * 2;
  static_assert(kBytes % (1024 * WAVES) == 0, "whole transfers, as many for each wavefront");
  uint32_t offset[kLoads];  // of this lane's pieces from the operand's first element of the stage
  int at_k[kLoads];         // their place along k
  static __device__ inline int turn(int k) {
    return P % 128 == 0 ? (k & 3) | (k >> 3 & 1) << 2 : (k >> 1 & 1) | (k >> 3 & 1) << 1;
  }

  __device__ inline void begin(const Source &s, int64_t p0, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int f = (i * WAVES + wave) * 64 + lane;
      if (K_LAST) {
        const int r = f / 8, c = (f % 8) ^ (r & 7);
        at_k[i] = c * 8;
        offset[i] = p0 + r < s.extent ? (uint32_t)(r * s.ld + c * 16) : kNowhere;
      } else {
        const int r = f / (P / 8), c = (f % (P / 8)) ^ (2 * turn(r));
        at_k[i] = r;
        offset[i] = p0 + c * 8 < s.extent ? (uint32_t)(r * s.ld + c * 16) : kNowhere;
      }
    }
  }
  // Where the first step's transfers read from, and how far apart the steps are.
  static __device__ inline uint64_t place(const Source &s, int64_t p0, int64_t step) {
    return (uint64_t)s.base + (K_LAST ? p0 * s.ld + step * (kStep * 2) : step * kStep * s.ld + p0 * 2);
  }
  static __device__ inline int64_t apart(const Source &s) { return K_LAST ? kStep * 2 : kStep * s.ld; }
  // Starts this wavefront's transfer `i` of the step at `from` into the stage at `lds`; `left`: what of k there is from the
  // step's first on, 0 and less where nothing is.
  __device__ inline void bring(int i, uint64_t from, int left, uint32_t lds, int wave) const {
    const u32x4 resource = {(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)from), (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(from >> 32)), kNowhere,
                            0x00020000u};
    to_lds(lds + (i * WAVES + wave) * 1024, at_k[i] < left ? offset[i] : kNowhere, resource);
  }
  // The operand of a matrix instruction: 16 lines from p (a multiple of 16) on, 32 of k from 32 * half on.
  static __device__ inline u32x4 read(const uint8_t *lds, int p, int half, int lane) {
    if (K_LAST) return *(const u32x4 *)(lds + (p + lane % 16) * 128 + ((half * 4 + lane / 16) ^ (lane & 7)) * 16);
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 *Place;
    const int k = half * 32 + lane / 16 * 8 + lane % 16 / 4;
    const uint8_t *at = lds + k * kLine + (((p / 16) ^ turn(k)) * 32) + lane % 4 * 8;
    const s16x4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Place)at), high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Place)(at + 4 * kLine));
    return __builtin_bit_cast(u32x4, __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// Tiles of (WM * MI * 16) x (WN * NI * 16), a wavefront has MI * 16 rows of NI * 16 columns.  STAGES stages of LDS, and the
// operands of two matrix instructions' k in registers: while those of one run, the other's come from LDS, and one stage is read
// while the others are filled.
template <typename T, int MI, int NI, int WM, int WN, int STAGES, bool A_K, bool B_K>
__global__ __launch_bounds__(WM *WN * 64, 2) void ds_matmul_tile_kernel(TileArgs t, Epilogue e) {
  constexpr int kWaves = WM * WN, kM = WM * MI * 16, kN = WN * NI * 16;
  typedef Stage<kM, kWaves, A_K> A;
  typedef Stage<kN, kWaves, B_K> B;
  constexpr int kStage = A::kBytes + B::kBytes, kOutPitch = NI * 16;
  // of 16 rows of the sums each, as many as the stages' LDS holds for every wavefront: all, or half of them
  constexpr int kRoom = STAGES * kStage / (kWaves * 16 * kOutPitch * 4), kOut = kRoom >= MI ? MI : MI / 2;
  static_assert(NI == 4 && kWaves * kOut * 16 * kOutPitch * 4 <= STAGES * kStage, "the sums leave through the stages");
  __shared__ __attribute__((aligned(1024))) uint8_t lds[STAGES * kStage];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // Work-groups go to the eight XCDs in turn: each XCD gets a run of neighbouring tiles, in stripes of four tiles' rows, so that
  // what its work-groups read at a time stays in its L2.
  const uint32_t tiles = t.tiles_m * t.tiles_n, all = tiles * t.splits, each = all / 8, more = all % 8;
  const uint32_t xcd = blockIdx.x % 8, id = xcd * each + (xcd < more ? xcd : more) + blockIdx.x / 8;
  const uint32_t split = id / tiles, tile = id % tiles, stripe = tile / (4 * t.tiles_n), in_stripe = tile % (4 * t.tiles_n);
  const uint32_t high = t.tiles_m - stripe * 4 < 4 ? t.tiles_m - stripe * 4 : 4;
  const int64_t p0 = (int64_t)(stripe * 4 + in_stripe % high) * kM, q0 = (int64_t)(in_stripe / high) * kN;

  const int64_t steps = (t.depth + kStep - 1) / kStep, first = steps * split / t.splits, last = steps * (split + 1) / t.splits;
  A a;
  B b;
  a.begin(t.a, p0, wave, lane);
  b.begin(t.b, q0, wave, lane);
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
  // The step whose transfers start next.
  uint64_t from_a = A::place(t.a, p0, first), from_b = B::place(t.b, q0, first);
  const int64_t apart_a = A::apart(t.a), apart_b = B::apart(t.b);
  int left = (int)((last * kStep < t.depth ? last * kStep : t.depth) - first * kStep);
  constexpr int kLoads = A::kLoads + B::kLoads;
  const auto bring = [&](int i, int to) {
    if (i < A::kLoads) a.bring(i, from_a, left, base + to * kStage, wave);
    else b.bring(i - A::kLoads, from_b, left, base + to * kStage + A::kBytes, wave);
    if (i == kLoads - 1) from_a += apart_a, from_b += apart_b, left -= kStep;
  };
  const int m0 = wave / WN * MI * 16, n0 = wave % WN * NI * 16;
  f32x4 sum[MI][NI] = {};
  struct Operands {
    u32x4 x[MI], y[NI];
  } even, odd;
  const auto fetch = [&](Operands &o, const uint8_t *stage, int half, int i) {
    if (i < NI) o.y[i] = B::read(stage + A::kBytes, n0 + i * 16, half, lane);
    else o.x[i - NI] = A::read(stage, m0 + (i - NI) * 16, half, lane);
  };
  // 32 of k on the operands in `now`, while the next 32's come from half `half` of the stage `next_at`; with the first half a later
  // step's transfers to the stage `to` start.  Reads and transfers stand between the matrix instructions: a wavefront that
  // starts all its transfers at once waits for the unit that takes them, 16 cycles for each.  (Transfers behind the last step
  // bring zeros.)
  constexpr int kQuiet = MI / 8;
  const auto advance = [&](const Operands &now, Operands &next, int next_at, auto half, int to) {
    const uint8_t *stage = lds + next_at * kStage;
    // rows of matrix instructions in front of the barrier, with it, and behind the last read
    constexpr int kFirst = half == 0 ? kQuiet : 0, kReading = MI - kFirst - kQuiet;
    int read = 0, brought = 0;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      if (half == 0 && i == kFirst) stage_is_there<(STAGES - 2) * kLoads>();
      if (i >= kFirst) {
#pragma unroll
        for (; read < MI + NI && read * kReading < (MI + NI) * (i + 1 - kFirst); ++read) fetch(next, stage, half, read);
#pragma unroll
        for (; half == 0 && brought * (MI - kFirst) < kLoads * (i + 1 - kFirst); ++brought) bring(brought, to);
      }
#pragma unroll
      for (int j = 0; j < NI; ++j) sum[i][j] = mfma(now.y[j], now.x[i], sum[i][j], T());
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  const auto after = [](int stage) { return stage + 1 == STAGES ? 0 : stage + 1; };
#pragma unroll
  for (int s = 0; s < STAGES; ++s)
#pragma unroll
    for (int i = 0; i < kLoads; ++i) bring(i, s);
  stage_is_there<(STAGES - 1) * kLoads>();
#pragma unroll
  for (int i = 0; i < MI + NI; ++i) fetch(even, lds, 0, i);
  // One barrier a step.  Behind it everybody has the step's second half in registers, so that its stage is free for the step
  // STAGES further on, and the next step's stage is there.
  int at = 0;
  for (int64_t step = first; step < last; ++step) {
    const int next = after(at);
    advance(even, odd, at, std::integral_constant<int, 1>(), 0);
    advance(odd, even, next, std::integral_constant<int, 0>(), at);
    at = next;
  }
  stage_is_there<0>();
  // a lane's sums: row lane % 16 of the 16, columns 16 j + 4 (lane / 16) and on
  if (t.partial) {
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int64_t row = p0 + m0 + i * 16 + lane % 16;
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int64_t col = q0 + n0 + j * 16 + lane / 16 * 4;
        float *to = t.partial + ((int64_t)split * e.m + row) * e.n + col;
        if (row < e.m)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (col + k < e.n) to[k] = sum[i][j][k];
      }
    }
    return;
  }
  // kRows of the wavefront's rows at a time go through LDS, and leave eight columns a lane, kBatch rows' residual asked for
  // before the first of them is finished.
  constexpr int kLanes = NI * 2, kPass = 64 / kLanes, kPasses = kOut * 16 / kPass, kBatch = kPasses % 4 == 0 ? 4 : kPasses % 3 == 0 ? 3 : kPasses % 2 == 0 ? 2 : 1;
  static_assert(MI % kOut == 0 && kPasses % kBatch == 0, "whole batches");
  float *out = (float *)lds + wave * kOut * 16 * kOutPitch;
  const int col = lane % kLanes * 8;
  // four floats, their place in a row exchanged by the row, so that 16 rows' are in different banks
  const auto piece = [](int row, int at) { return (at ^ (row & 15)) * 4; };
  const int64_t j = q0 + n0 + col;
  const Eight bias = bias8(e, j, columns_of(e, 0, j));
  // (The registers that hold the sums are named in the code, so each part's way to LDS is written out; the rest is one loop.)
  const auto leave = [&](auto type, auto whole) {
    typedef decltype(type) C;
#pragma unroll 1
    for (int h = 0; h < MI / kOut; ++h) {
#pragma unroll
      for (int part = 0; part < MI / kOut; ++part)
        if (h == part) {
#pragma unroll
          for (int i = 0; i < kOut; ++i)
#pragma unroll
            for (int b = 0; b < NI; ++b) *(f32x4 *)(out + (i * 16 + lane % 16) * kOutPitch + piece(lane, b * 4 + lane / 16)) = sum[part * kOut + i][b];
        }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll 1
      for (int pass = 0; pass < kPasses; pass += kBatch) {
        typename RowsOf<C>::Bits residual[kBatch];
        const int64_t row0 = p0 + m0 + h * kOut * 16 + pass * kPass + lane / kLanes;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) residual[u] = residual8<C>(e, row0 + u * kPass, j, whole ? 8 : columns_of(e, row0 + u * kPass, j));
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int row = (pass + u) * kPass + lane / kLanes;
          Eight z;
          const f32x4 lo = *(const f32x4 *)(out + row * kOutPitch + piece(row, col / 4)), hi = *(const f32x4 *)(out + row * kOutPitch + piece(row, col / 4 + 1));
#pragma unroll
          for (int k = 0; k < 4; ++k) z.v[k] = lo[k], z.v[4 + k] = hi[k];
          finish8<C>(e, row0 + u * kPass, j, whole ? 8 : columns_of(e, row0 + u * kPass, j), z, bias, residual[u]);
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  };
  with_c_type(e, [&](auto type) {
    if (p0 + kM <= e.m && q0 + kN <= e.n) leave(type, std::true_type());
    else leave(type, std::false_type());
  });
}

// The sums of the splits, in their order, and the epilogue.  A row has a multiple of four pieces of eight columns.
template <typename C, typename Index>
__global__ __launch_bounds__(kThreads) void ds_matmul_join_kernel(const float *partial, uint32_t splits, uint32_t pieces, Epilogue e) {
  for (int64_t first = (int64_t)blockIdx.x * kThreads; first < e.m * pieces; first += (int64_t)gridDim.x * kThreads) {
    const Index item = (Index)(first + threadIdx.x), row = item / (Index)pieces;
    const int64_t i = row, j = (int64_t)(item - row * (Index)pieces) * 8;
    const int n = columns_of(e, i, j);
    const auto residual = residual8<C>(e, i, j, n);
    const float *from = partial + i * e.n + j;
    const int64_t apart = e.m * e.n;
    Eight z = {};
    uint32_t s = 0;
    for (; s + 4 <= splits; s += 4, from += 4 * apart) {  // four at a time on their way
      Eight p[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) p[u] = get_up_to8<float>(from, u * apart, n);
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int k = 0; k < 8; ++k) z.v[k] += p[u].v[k];
    }
    for (; s < splits; ++s, from += apart) {
      const Eight p = get_up_to8<float>(from, 0, n);
#pragma unroll
      for (int k = 0; k < 8; ++k) z.v[k] += p.v[k];
    }
    finish8<C>(e, i, j, n, z, bias8(e, j, n), residual);
  }
}

// An operand's lines of `length` elements as lines of 16-bit values, a multiple of eight of them, the rest zeros.  Bound by HBM: a checkpoint
// of 16384 x 4096 is read and written in 37 us, 5.4 TB/s, beside 320 us of the product that it goes into.  (Making
// 16-bit values of the codes in the tiles' kernel would do it once for every row of tiles.)
template <typename T, typename Index>
__global__ __launch_bounds__(kThreads) void ds_matmul_lines_kernel(Operand o, int64_t lines, int64_t length, uint16_t *out, uint32_t pieces) {
  for (int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x; at < lines * pieces; at += (int64_t)gridDim.x * kThreads) {
    const Index line = (Index)at / (Index)pieces;
    const int64_t j = (int64_t)((Index)at - line * (Index)pieces) * 8;
    *(u32x4 *)(out + at * 8) = o.k_last ? bring8<T>(o, line, j, length) : bring8<T>(o, j, line, lines);
  }
}

// ---- few rows of a, and a weight [out, in] -------------------------------------------------------------------------

// At most 16 rows: what counts is reading b once, at the rate of HBM.  A work-group of eight wavefronts has 16 or 32 columns of c; a wavefront
// takes every eighth piece of 64 k, so that neighbouring wavefronts read neighbouring lines, and asks for the next four pieces
// before it multiplies these.  A lane reads 32 neighbouring bytes of a line of b, two matrix instructions' operands: the order of k within
// a piece is any, as long as a's is the same.  The wavefronts' sums are added in their order, in LDS.
constexpr int kFewWaves = 8;

// Eight neighbouring k of line p from k on; what is beyond the matrix is 0.
__device__ inline u32x4 line8(const Operand &o, int64_t p, int64_t k, int64_t depth) {
  u32x4 r = {0, 0, 0, 0};
  if (p >= o.extent) return r;
  const uint16_t *q = (const uint16_t *)o.base + p * o.ld + k;
  if (k + 8 <= depth) return *(const ds_u32x4 *)q;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (k + i < depth) r[i / 2] |= (uint32_t)q[i] << (16 * (i % 2));
  return r;
}

template <typename T, int SETS>
__global__ __launch_bounds__(kFewWaves * 64) void ds_matmul_few_kernel(Operand a, Operand b, Epilogue e, int64_t depth) {
  constexpr int kPieces = 4, kFewCols = SETS * 16;
  __shared__ float sums[kFewWaves][kFewRows][kFewCols + 4];
  __shared__ float out[kFewRows][kFewCols + 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, line = lane % 16;
  const int64_t q0 = (int64_t)blockIdx.x * kFewCols;
  f32x4 sum[SETS] = {};
  struct Piece {
    u32x4 w[SETS][2], x[2];
  };
  // lines beyond the matrix read its last one, and lead to sums that nobody stores
  const uint16_t *from_w[SETS], *from_x;
#pragma unroll
  for (int s = 0; s < SETS; ++s) {
    const int64_t p = q0 + s * 16 + line;
    from_w[s] = (const uint16_t *)b.base + (p < b.extent ? p : b.extent - 1) * b.ld + lane / 16 * 16;
  }
  from_x = (const uint16_t *)a.base + (line < a.extent ? line : a.extent - 1) * a.ld + lane / 16 * 16;
  const auto ask = [&](Piece &p, int64_t k) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int s = 0; s < SETS; ++s) p.w[s][h] = *(const ds_u32x4 *)(from_w[s] + k + h * 8);
      p.x[h] = *(const ds_u32x4 *)(from_x + k + h * 8);
    }
  };
  const auto multiply = [&](const Piece &p) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int s = 0; s < SETS; ++s) sum[s] = mfma(p.w[s][h], p.x[h], sum[s], T());
  };
  constexpr int64_t kApart = kFewWaves * 64;
  // this wavefront's whole pieces, the first `fours` of them four at a time
  const int64_t whole = depth / 64, mine = whole > wave ? (whole - wave + kFewWaves - 1) / kFewWaves : 0, fours = mine / kPieces;
  int64_t k = wave * 64;
  if (fours > 0) {
    Piece now[kPieces], next[kPieces];
#pragma unroll
    for (int u = 0; u < kPieces; ++u) ask(now[u], k + u * kApart);
    for (int64_t f = 1; f < fours; ++f) {
      k += kPieces * kApart;
#pragma unroll
      for (int u = 0; u < kPieces; ++u) ask(next[u], k + u * kApart);
#pragma unroll
      for (int u = 0; u < kPieces; ++u) multiply(now[u]), now[u] = next[u];
    }
#pragma unroll
    for (int u = 0; u < kPieces; ++u) multiply(now[u]);
    k += kPieces * kApart;
  }
  for (int64_t f = fours * kPieces; f < mine; ++f, k += kApart) {
    Piece p;
    ask(p, k);
    multiply(p);
  }
  if (depth % 64 != 0 && whole % kFewWaves == wave) {  // the rest of k
    Piece p;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t at = whole * 64 + lane / 16 * 16 + h * 8;
#pragma unroll
      for (int s = 0; s < SETS; ++s) p.w[s][h] = line8(b, q0 + s * 16 + line, at, depth);
      p.x[h] = line8(a, line, at, depth);
    }
    multiply(p);
  }
  // a lane's sums: row lane % 16, columns 16 s + 4 (lane / 16) and on
#pragma unroll
  for (int s = 0; s < SETS; ++s) *(f32x4 *)&sums[wave][line][s * 16 + lane / 16 * 4] = sum[s];
  __syncthreads();
  if (threadIdx.x < kFewRows * kFewCols) {
    const int i = threadIdx.x / kFewCols, j = threadIdx.x % kFewCols;
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) total += sums[w][i][j];
    out[i][j] = total;
  }
  __syncthreads();
  if (wave != 0) return;
  with_c_type(e, [&](auto type) {
    typedef decltype(type) C;
    const int64_t i = lane / (SETS * 2), j = q0 + lane % (SETS * 2) * 8;
    const int n = i < kFewRows ? columns_of(e, i, j) : 0;
    Eight z = {};
    if (n > 0)
#pragma unroll
      for (int k = 0; k < 8; ++k) z.v[k] = out[i][lane % (SETS * 2) * 8 + k];
    finish8<C>(e, i, j, n, z, bias8(e, j, n), residual8<C>(e, i, j, n));
  });
}

int check_product(const ds_matrix *a, const ds_matrix *b, const ds_matrix *c) {
  DS_TRY(ds_check_matrix(a, false));
  DS_TRY(ds_check_matrix(b, false));
  DS_TRY(ds_check_matrix(c, true));
  const bool a8 = a->dtype == DS_MX8, b8 = b->dtype == DS_MX8;
  if ((!a8 && !ds_is_half(a->dtype)) || (!b8 && !ds_is_half(b->dtype)) || (!a8 && !b8 && a->dtype != b->dtype) || c->dtype == DS_MX8 ||
      a->cols != b->rows || a->rows != c->rows || b->cols != c->cols)
    return DS_EINVAL;
  return DS_OK;
}

// ---- launches -------------------------------------------------------------------------------------------------------

int launch_join(const float *partial, uint32_t splits, const Epilogue &e, hipStream_t stream) {
  const int64_t pieces = ds_groups(e.n) * (kGroup / 8), groups = (e.m * pieces + kThreads - 1) / kThreads;
  return ds_with_type(e.c_dtype, [&](auto type) -> int {
    typedef decltype(type) C;
    const auto launch = [&](auto kernel) -> int {
      hipLaunchKernelGGL(kernel, dim3((uint32_t)(groups < kMaxGrid ? groups : kMaxGrid)), dim3(kThreads), 0, stream, partial, splits,
                         (uint32_t)pieces, e);
      DS_HIP_TRY(hipGetLastError());
      return DS_OK;
    };
    return groups <= (int64_t)0xffffffff / kThreads ? launch(ds_matmul_join_kernel<C, uint32_t>) : launch(ds_matmul_join_kernel<C, uint64_t>);
  });
}

template <typename T>
int launch_lines(const Operand &o, int64_t depth, uint8_t *out, Source *s, hipStream_t stream) {
  const int64_t lines = o.k_last ? o.extent : depth, length = o.k_last ? depth : o.extent, pieces = (length + 7) / 8;
  const int64_t groups = (lines * pieces + kThreads - 1) / kThreads;
  const auto launch = [&](auto kernel) -> int {
    hipLaunchKernelGGL(kernel, dim3((uint32_t)(groups < kMaxGrid ? groups : kMaxGrid)), dim3(kThreads), 0, stream, o, lines, length,
                       (uint16_t *)out, (uint32_t)pieces);
    DS_HIP_TRY(hipGetLastError());
    return DS_OK;
  };
  DS_TRY(groups <= (int64_t)0xffffffff / kThreads ? launch(ds_matmul_lines_kernel<T, uint32_t>) : launch(ds_matmul_lines_kernel<T, uint64_t>));
  // (the zeros behind a line of p are columns of no output)
  *s = Source{out, pieces * 16, o.k_last ? o.extent : pieces * 8};
  return DS_OK;
}

template <typename T, int MI, int NI, int WM, int WN, int STAGES>
int launch_tile(const Operand &a, const Operand &b, const TileArgs &t, const Epilogue &e, hipStream_t stream) {
  const dim3 grid(t.tiles_m * t.tiles_n * t.splits), threads(WM * WN * 64);
  if (a.k_last && b.k_last) hipLaunchKernelGGL((ds_matmul_tile_kernel<T, MI, NI, WM, WN, STAGES, true, true>), grid, threads, 0, stream, t, e);
  else if (a.k_last) hipLaunchKernelGGL((ds_matmul_tile_kernel<T, MI, NI, WM, WN, STAGES, true, false>), grid, threads, 0, stream, t, e);
  else if (b.k_last) hipLaunchKernelGGL((ds_matmul_tile_kernel<T, MI, NI, WM, WN, STAGES, false, true>), grid, threads, 0, stream, t, e);
  else hipLaunchKernelGGL((ds_matmul_tile_kernel<T, MI, NI, WM, WN, STAGES, false, false>), grid, threads, 0, stream, t, e);
  DS_HIP_TRY(hipGetLastError());
  return DS_OK;
}

template <typename T>
int launch_product(const Operand &a, const Operand &b, const Epilogue &e, int64_t depth, const Choice &c, uint8_t *ws, hipStream_t stream) {
  if (c.way == Way::kSimple) {
    const int64_t across = (e.n + kTile - 1) / kTile, down = (e.m + kTile - 1) / kTile;
    hipLaunchKernelGGL(ds_matmul_kernel<T>, dim3((uint32_t)(across * down)), dim3(kThreads), 0, stream, a, b, e, depth, (uint32_t)across);
    DS_HIP_TRY(hipGetLastError());
    return DS_OK;
  }
  if (c.way == Way::kFew) {
    // 16 columns a work-group while those of 32 would leave CUs without one; a checkpoint's groups are 32
    if (e.n <= 32 * kCus && !e.saved.base)
      hipLaunchKernelGGL((ds_matmul_few_kernel<T, 1>), dim3((uint32_t)((e.n + 15) / 16)), dim3(kFewWaves * 64), 0, stream, a, b, e, depth);
    else
      hipLaunchKernelGGL((ds_matmul_few_kernel<T, 2>), dim3((uint32_t)((e.n + 31) / 32)), dim3(kFewWaves * 64), 0, stream, a, b, e, depth);
    DS_HIP_TRY(hipGetLastError());
    return DS_OK;
  }
  const TileSize &s = kTiles[c.tile];
  TileArgs t{{(const uint8_t *)a.base, a.ld * 2, a.extent}, {(const uint8_t *)b.base, b.ld * 2, b.extent}, depth,
             (uint32_t)((e.m + s.m - 1) / s.m), (uint32_t)((e.n + s.n - 1) / s.n), c.splits, c.splits > 1 ? (float *)(ws + c.at_partial) : nullptr};
  if (c.lines_a) DS_TRY(launch_lines<T>(a, depth, ws + c.at_a, &t.a, stream));
  if (c.lines_b) DS_TRY(launch_lines<T>(b, depth, ws + c.at_b, &t.b, stream));
  switch (c.tile) {
    case 0: DS_TRY((launch_tile<T, 8, 4, 2, 4, 2>(a, b, t, e, stream))); break;
    case 1: DS_TRY((launch_tile<T, 6, 4, 2, 4, 2>(a, b, t, e, stream))); break;
    case 2: DS_TRY((launch_tile<T, 4, 4, 2, 4, 3>(a, b, t, e, stream))); break;
    case 3: DS_TRY((launch_tile<T, 2, 4, 4, 2, 3>(a, b, t, e, stream))); break;
    case 4: DS_TRY((launch_tile<T, 2, 4, 2, 2, 3>(a, b, t, e, stream))); break;
    default: DS_TRY((launch_tile<T, 1, 4, 4, 1, 3>(a, b, t, e, stream))); break;
  }
  if (c.splits == 1) return DS_OK;
  return launch_join(t.partial, t.splits, e, stream);
}

}  // namespace

extern "C" int ds_matmul_workspace(const ds_matrix *a, const ds_matrix *b, const ds_matrix *c, uint64_t *bytes) {
  if (!bytes) return DS_EINVAL;
  DS_TRY(check_product(a, b, c));
  const Choice how = choose(operand(a, true), operand(b, false), c->rows, c->cols, a->cols);
  if (how.way == Way::kNone) return DS_ERANGE;
  *bytes = how.bytes;
  return DS_OK;
}

extern "C" int ds_matmul(const ds_matrix *a, const ds_matrix *b, const ds_matrix *c, const ds_matmul_epilogue *epilogue, void *workspace,
                         uint64_t workspace_bytes, void *stream) {
  DS_TRY(check_product(a, b, c));
  static const ds_matmul_epilogue nothing = {nullptr, DS_F32, DS_ACT_NONE, nullptr, nullptr};
  const ds_matmul_epilogue &ep = epilogue ? *epilogue : nothing;
  if (ep.act > DS_ACT_SILU || (ep.bias && (!ds_is_float(ep.bias_dtype) || ds_misaligned(ep.bias, ds_itemsize(ep.bias_dtype))))) return DS_EINVAL;
  if (ep.residual) {
    DS_TRY(ds_check_matrix(ep.residual, true));
    if (ep.residual->dtype != c->dtype || !ds_same_extents(ep.residual, c)) return DS_EINVAL;
  }
  if (ep.saved) {
    DS_TRY(ds_check_matrix(ep.saved, true));
    if (ep.saved->dtype != DS_MX8 || !ds_same_extents(ep.saved, c)) return DS_EINVAL;
  }
  if (c->rows == 0 || c->cols == 0) return DS_OK;
  const Operand oa = operand(a, true), ob = operand(b, false);
  const Choice how = choose(oa, ob, c->rows, c->cols, a->cols);
  if (how.way == Way::kNone) return DS_ERANGE;
  if (how.bytes) {
    if (!workspace || ds_misaligned(workspace, 16)) return DS_EINVAL;
    if (workspace_bytes < how.bytes) return DS_ERANGE;
  }
  const Epilogue e{ds_rows(c), ds_rows(ep.residual), ds_rows(ep.saved), ep.bias, c->rows, c->cols, c->dtype, ep.bias_dtype, ep.act};
  if (a->dtype == DS_F16 || b->dtype == DS_F16)
    return launch_product<__half>(oa, ob, e, a->cols, how, (uint8_t *)workspace, (hipStream_t)stream);
  return launch_product<__hip_bfloat16>(oa, ob, e, a->cols, how, (uint8_t *)workspace, (hipStream_t)stream);
}
