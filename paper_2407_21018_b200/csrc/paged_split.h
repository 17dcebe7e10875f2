// How the flat tile list of a paged attention call is cut: N tiles over `grid` CTAs, a CTA's tiles over its warps.
// Plain integer arithmetic, shared with the host's tests.
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
// part i of n tiles cut into `parts`: [split_begin(i), split_begin(i + 1)); n * parts fits 62 bits
THINK_HD int64_t split_begin(int64_t n, int parts, int i) { return div_wide((int64_t)i * n, parts); }
// the part that owns tile f, 0 <= f < n
THINK_HD int split_owner(int64_t n, int parts, int64_t f) { return (int)div_wide((f + 1) * parts - 1, n); }

}  // namespace think
