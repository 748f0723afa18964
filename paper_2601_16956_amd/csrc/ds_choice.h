// How ds_matmul computes a product: host arithmetic on sizes, strides and alignment, without a device.
#pragma once

#include <stdint.h>

#include "datastates.h"

namespace {

// An operand: element (p, k), p a row of a or a column of b.
struct Operand {
  const void *base;
  int64_t ld;      // elements from p to p + 1 (k_last), or from k to k + 1
  int64_t extent;  // of p
  const uint8_t *scale;
  int64_t scale_stride;
  bool k_last;  // neighbouring k are neighbours in memory
};

// a (or b's transpose): p along `along` = its rows if `p_rows`.
inline Operand operand(const ds_matrix *m, bool p_rows) {
  const int64_t p = p_rows ? m->rows : m->cols, k = p_rows ? m->cols : m->rows;
  const int64_t step_p = p_rows ? m->row_stride : m->col_stride, step_k = p_rows ? m->col_stride : m->row_stride;
  // in rows if the columns are neighbours; a matrix of one row or column may be either
  const bool in_rows = (m->cols <= 1 || m->col_stride == 1) && (m->rows <= 1 || m->row_stride >= m->cols);
  const bool k_last = in_rows == p_rows;
  const int64_t ld = k_last ? (p > 1 ? step_p : k) : (k > 1 ? step_k : p);
  return Operand{m->base, ld, p, m->dtype == DS_MX8 ? m->scale : nullptr, m->scale_stride, k_last};
}

constexpr int kStep = 64;  // of k: what a stage of LDS holds, twice what a matrix instruction takes
constexpr int kFewRows = 16;  // rows of a that the kernel for few rows takes

constexpr int64_t kMaxTiles = 1 << 22;  // work-groups of a launch

enum class Way { kSimple, kTile, kFew, kNone };  // kNone: there are too many tiles for any
struct Choice {
  Way way;
  int tile;         // index into kTiles
  uint32_t splits;
  bool lines_a, lines_b;  // is the operand laid out in the workspace first?
  uint64_t at_a, at_b, at_partial, bytes;
};
// A tile's extents, how many of its work-groups a CU holds, and what they take, in us: before and behind the steps; a step where most
// CUs are idle; a step with 1, 2, 3 work-groups on every CU.  (Measured with bfloat16 [out, in] on products of 4 to 256 steps; what
// the steps take on a full chip is decided by its power.  Neither the epilogue is in them, nor laying out lines, nor memory that cannot
// follow: 515 x 1000 x 777 is put at 9 us and takes 12, and 4 for the lines.)
struct TileSize {
  int m, n, at_once;
  double around, idle, step[3];
};
constexpr TileSize kTiles[] = {
    {256, 256, 1, 9.9, 0.96, {1.41}},       {192, 256, 1, 8.6, 0.78, {1.20}},
    {128, 256, 1, 7.1, 0.56, {0.80}},       {128, 128, 1, 5.6, 0.36, {0.55}},
    {64, 128, 2, 5.2, 0.295, {0.33, 0.66}}, {64, 64, 3, 4.7, 0.255, {0.27, 0.36, 0.70}},
};
constexpr int64_t kCus = 256;
inline int64_t tiles_of(int64_t m, int64_t n, int64_t tile_m, int64_t tile_n) { return (m + tile_m - 1) / tile_m * ((n + tile_n - 1) / tile_n); }
inline double tile_time(const TileSize &s, int64_t tiles, int64_t m, int64_t n, int64_t steps, int64_t splits) {
  const int64_t groups = tiles * splits, each = (steps + splits - 1) / splits;
  const int64_t on_cu = (groups + kCus - 1) / kCus, rounds = (on_cu + s.at_once - 1) / s.at_once, rest = on_cu % s.at_once;
  double step = (double)(on_cu / s.at_once) * s.step[s.at_once - 1] + (rest ? s.step[rest - 1] : 0.0);
  if (on_cu == 1) step = s.idle + (s.step[0] - s.idle) * (double)groups / kCus;
  // a further round's beginning and end; those of work-groups that share a CU overlap
  double t = s.around + (double)each * step + (double)(rounds - 1) * (s.around - 3.0);
  if (splits > 1) t += 4.0 + (double)m * (double)n * (double)splits * 8.0 / 5e6;  // the sums' way through memory, and a launch
  return t;
}

// May the operand be read in 16-byte pieces, all within its lines?
inline bool in_pieces(const Operand &o, int64_t depth) {
  const int64_t length = o.k_last ? depth : o.extent;
  return !o.scale && ((uintptr_t)o.base & 15) == 0 && length % 8 == 0 && (o.ld % 8 == 0) && o.ld < (1 << 21);
}
inline uint64_t lines_bytes(const Operand &o, int64_t depth) {
  const int64_t lines = o.k_last ? o.extent : depth, length = o.k_last ? depth : o.extent;
  return ((uint64_t)lines * (uint64_t)((length + 7) / 8 * 8) * 2 + 127) / 128 * 128;
}

// At most 16 rows on lines along k: does the kernel for them take the product, or the tiles?  It reads b once and joins nothing, but each of
// its work-groups walks along all of k, and with n <= 2048 there are few of them; tiles split k.  And where k is short and n long
// its work-groups, one a CU, come in several rounds.  us of the GPU, it / tiles, bfloat16, 1 and 16 rows:
//      k     n = 64      n = 1024     n = 2048     n = 4096     n = 8192    n = 16384    n = 28672
//    512   7.1/14  4/6   4.2/6  5/6   4.0/6  4/6   4.3/7  5/7   5.9/7  7/7   7.8/7  8/7   13/9  14/10
//   4096   7.5/10 10/9   8.0/10 11/10 8.1/11 11/12 8.9/13 11/13 17/19 23/20  31/39 33/40  52/52 58/54
//   8192    12/11 17/10   12/11 18/12  13/13 18/14  17/20 22/21 30/39 40/41  63/66 64/68  109/104 115/104
//  16384    21/13 31/12   22/14 32/15  23/22 33/23  32/65 37/67 60/115 68/111 108/179 101/174 195/199 191/199
// (Elsewhere, n = 6144 and 12288 with k >= 4096, either is up to 25 % ahead; this kernel has them.)
inline bool few_rows(int64_t m, int64_t n, int64_t depth) {
  if (m > kFewRows || n > kMaxTiles * 32) return false;
  if (n <= 2048) return depth <= 7000 - 200 * m + 2 * (n > 1024 ? n - 1024 : 0);
  return n <= 8192 || depth >= 1024;
}

inline Choice choose(const Operand &a, const Operand &b, int64_t m, int64_t n, int64_t depth) {
  Choice c{tiles_of(m, n, 64, 64) <= kMaxTiles ? Way::kSimple : Way::kNone, 0, 1, false, false, 0, 0, 0, 0};
  // lines of 16-bit values are at most 2^22 bytes apart, so that a stage's offsets have 31 bits
  const auto too_long = [&](const Operand &o) { return (o.k_last ? depth : o.extent) > (1 << 21); };
  if (depth == 0) return c;
  if (a.k_last && b.k_last && !a.scale && !b.scale && few_rows(m, n, depth)) {
    c.way = Way::kFew;
    return c;
  }
  if ((double)m * (double)n * (double)depth < (1 << 18) || too_long(a) || too_long(b)) return c;
  const int64_t steps = (depth + kStep - 1) / kStep;
  double best = 1e300;
  for (int i = 0; i < (int)(sizeof kTiles / sizeof kTiles[0]); ++i) {
    const int64_t tiles = tiles_of(m, n, kTiles[i].m, kTiles[i].n);
    for (int64_t splits = 1; splits <= 16 && splits * 4 <= steps + 3 && tiles * splits <= kMaxTiles; ++splits) {
      const double time = tile_time(kTiles[i], tiles, m, n, steps, splits);
      if (time < best) best = time, c.way = Way::kTile, c.tile = i, c.splits = (uint32_t)splits;
    }
  }
  if (c.way != Way::kTile) return c;
  c.lines_a = !in_pieces(a, depth), c.lines_b = !in_pieces(b, depth);
  if (c.lines_a) c.at_a = c.bytes, c.bytes += lines_bytes(a, depth);
  if (c.lines_b) c.at_b = c.bytes, c.bytes += lines_bytes(b, depth);
  if (c.splits > 1) c.at_partial = c.bytes, c.bytes += (uint64_t)c.splits * m * n * 4;
  return c;
}

}  // namespace
