// Host build of how a product is computed (csrc/ds_choice.h, included unchanged).
#include "ds_choice.h"

// out: the way (0 simple, 1 tiles, 2 few rows), the tile's rows and columns, the splits, whether a and b are laid out first, the
// workspace's bytes.
extern "C" void choice_host(const ds_matrix *a, const ds_matrix *b, int64_t m, int64_t n, uint64_t *out) {
  const Choice c = choose(operand(a, true), operand(b, false), m, n, a->cols);
  out[0] = (uint64_t)c.way;
  out[1] = c.way == Way::kTile ? (uint64_t)kTiles[c.tile].m : 0;
  out[2] = c.way == Way::kTile ? (uint64_t)kTiles[c.tile].n : 0;
  out[3] = c.splits;
  out[4] = c.lines_a;
  out[5] = c.lines_b;
  out[6] = c.bytes;
}
