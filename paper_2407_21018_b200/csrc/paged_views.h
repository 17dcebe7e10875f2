// Whether the rows of strided destination views share memory.  Plain integer arithmetic, shared with the host's tests.
//
// Two rows share memory if the difference of their places is less than a row, so the question is whether an integer
// combination of the strides, each coefficient within its extent, falls into an interval.  The search takes the largest
// stride first and only the coefficients from which the smaller strides can still reach the interval: for views of dense
// tensors, sliced and permuted in any way, these are one to three a dimension.
#pragma once
#include <stdint.h>

namespace think {

struct StrideTerm {
  int64_t stride, lo, hi;      // coefficients lo .. hi
};

struct StrideSearch {
  StrideTerm t[8];
  int n = 0;
  int64_t steps = 0;
  static constexpr int64_t kMaxSteps = 1 << 16;      // more is taken for sharing: no call should wait for the answer

  // a dimension's coefficients; equal strides are one term, no stride is no term
  void add(int64_t stride, int64_t lo, int64_t hi) {
    if (stride == 0 || (lo == 0 && hi == 0)) return;
    int i = 0;
    while (i < n && t[i].stride > stride) ++i;
    if (i < n && t[i].stride == stride) {
      t[i].lo += lo;
      t[i].hi += hi;
      return;
    }
    for (int j = n++; j > i; --j) t[j] = t[j - 1];
    t[i] = StrideTerm{stride, lo, hi};
  }
  // is there a sum of the terms from i on in [lo, hi]
  bool hits(int64_t lo, int64_t hi, int i = 0) {
    if (++steps > kMaxSteps) return true;
    if (i == n) return lo <= 0 && hi >= 0;
    int64_t least = 0, most = 0;                      // of the terms behind this one
    for (int j = i + 1; j < n; ++j) {
      least += t[j].lo * t[j].stride;
      most += t[j].hi * t[j].stride;
    }
    const int64_t s = t[i].stride;
    int64_t c0 = floor_div(lo - most + s - 1, s), c1 = floor_div(hi - least, s);
    if (c0 < t[i].lo) c0 = t[i].lo;
    if (c1 > t[i].hi) c1 = t[i].hi;
    for (int64_t c = c0; c <= c1; ++c)
      if (hits(lo - c * s, hi - c * s, i + 1)) return true;
    return false;
  }
  static int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b < 0); }
};

// Rows of `row` units at the places sum of index * stride, index < extent; four dimensions, strides >= 0.  `spread`
// below 2^57 units (a view that spans more is no memory) keeps the sums above in 64 bits.
struct RowView {
  int64_t stride[4], extent[4], row;
  bool spread_ok() const {
    for (int i = 0; i < 4; ++i)
      if (extent[i] > 1 && stride[i] > ((int64_t)1 << 55) / (extent[i] - 1)) return false;
    return true;
  }
  bool shares_with_itself() const {
    for (int i = 0; i < 4; ++i)
      if (extent[i] > 1 && stride[i] < row) return true;               // neighbours
    // the first index that differs grows (in an order of the dimensions: the other half are mirror images)
    for (int i = 0; i < 4; ++i) {
      if (extent[i] <= 1) continue;
      StrideSearch q;
      for (int j = i + 1; j < 4; ++j) q.add(stride[j], 1 - extent[j], extent[j] - 1);
      q.add(stride[i], 1, extent[i] - 1);
      if (q.hits(1 - row, row - 1)) return true;
    }
    return false;
  }
  // the other view begins `apart` units behind this one
  bool shares_with(const RowView& o, int64_t apart) const {
    int64_t most = 0, other = 0;
    for (int i = 0; i < 4; ++i) {
      most += (extent[i] - 1) * stride[i];
      other += (o.extent[i] - 1) * o.stride[i];
    }
    if (apart > most + row - 1 || apart < -(other + o.row - 1)) return false;          // side by side: the usual case
    StrideSearch q;
    for (int i = 0; i < 4; ++i) {
      q.add(stride[i], 0, extent[i] - 1);
      q.add(o.stride[i], 1 - o.extent[i], 0);
    }
    return q.hits(apart - row + 1, apart + o.row - 1);
  }
};

}  // namespace think
