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

// part i of n tiles cut into `parts`: [split_begin(i), split_begin(i + 1)); n * parts fits 62 bits
THINK_HD int64_t split_begin(int64_t n, int parts, int i) { return (int64_t)i * n / parts; }
// the part that owns tile f, 0 <= f < n
THINK_HD int split_owner(int64_t n, int parts, int64_t f) { return (int)(((f + 1) * parts - 1) / n); }

}  // namespace think
