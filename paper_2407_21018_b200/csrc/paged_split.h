// How the tiles of a paged attention call are cut over CTAs and warps.  Plain integer arithmetic, shared with the
// host's tests.
//
// A unit (entry, layer, key head) of nt tiles takes tile * nt + unit places on a line: starting and ending a unit costs
// time too.  Tile j stands at slot(j) of its unit's places.  The line is cut evenly, and a part owns the tiles that
// stand in it.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define THINK_HD __host__ __device__ __forceinline__
#else
#define THINK_HD inline
#endif

namespace think {

// a / b, through the 32-bit division where both fit (a 64-bit one is a routine of a hundred instructions)
THINK_HD int64_t div_wide(int64_t a, int64_t b) {
  return (uint64_t)(a | b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}
// part i of n places cut into `parts`: [split_begin(i), split_begin(i + 1)); n * parts fits 62 bits
THINK_HD int64_t split_begin(int64_t n, int parts, int i) { return div_wide((int64_t)i * n, parts); }
// the part that holds place f, 0 <= f < n
THINK_HD int split_owner(int64_t n, int parts, int64_t f) { return (int)div_wide((f + 1) * parts - 1, n); }

struct Weights {
  int tile, unit;
  THINK_HD int cost(int nt) const { return tile * nt + unit; }
  THINK_HD int tiles(int cost) const { return (cost - unit) / tile; }
  // where tile j stands, and the first tile that stands at x or behind (may be none: nt or more)
  THINK_HD int slot(int j) const { return j == 0 ? 0 : unit + tile * j; }
  THINK_HD int first_tile(int64_t x) const {
    if (x <= 0) return 0;
    const int64_t j = (x - unit + tile - 1) / tile;
    return j < 1 ? 1 : j > 0x7fffffff ? 0x7fffffff : (int)j;
  }
};
// The weights `w`, or (1, 0) where there are too few tiles to weigh: any tile + unit neighbouring places hold a tile's,
// so no part of that many is without one.
THINK_HD Weights weights_for(Weights w, int64_t tiles, int64_t units, int parts) {
  return w.tile * tiles + w.unit * units >= (int64_t)(w.tile + w.unit) * parts ? w : Weights{1, 0};
}

}  // namespace think
