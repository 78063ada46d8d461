// Whether rows of two tensors share memory: for operators whose blocks read some rows while others are written.  Host only.
#pragma once
#include <stdint.h>

namespace stand {

// Rows of `bytes` bytes each at `at` and all sums of multiples (below count) of the strides (bytes, >= 0).
struct RowSet {
  const void* at;
  int64_t bytes;
  int dims;
  int64_t count[4], stride[4];
};

inline bool same_rows(const RowSet& x, const RowSet& y) {
  bool same = x.at == y.at && x.bytes == y.bytes && x.dims == y.dims;
  for (int i = 0; same && i < x.dims; ++i) same = x.count[i] == y.count[i] && (x.count[i] < 2 || x.stride[i] == y.stride[i]);
  return same;
}

// Two rows meet where a difference of their addresses, offset + sum of n_i stride_i with n_i in [lo_i, hi_i], lies between the rows' lengths.  A stride that
// both have in the same place is one such term, so rows that lie between others (queries beside keys in one projection) cost
// no more than a few steps.  Strides are taken from the largest down; where each covers the smaller ones there are two
// values to try for a term at most.  Layouts that take more than `steps` are not decided: false.
inline bool rows_meet(const RowSet& x, const RowSet& y) {
  using wide = __int128;
  const auto end = [](const RowSet& r) {
    wide e = (wide)(uintptr_t)r.at + r.bytes;
    for (int i = 0; i < r.dims; ++i) e += (wide)(r.count[i] - 1) * r.stride[i];
    return e;
  };
  if ((wide)(uintptr_t)x.at >= end(y) || (wide)(uintptr_t)y.at >= end(x)) return false;  // as most are
  struct Term {
    wide stride, lo, hi, below, above;  // below, above: what the terms after this one can add
  } t[8];
  int n = 0;
  auto add = [&](int64_t stride, int64_t lo, int64_t hi) {
    if (stride == 0 || lo == hi) return;
    int at = n++;
    for (; at > 0 && t[at - 1].stride < stride; --at) t[at] = t[at - 1];
    t[at] = {stride, lo, hi, 0, 0};
  };
  for (int i = 0; i < x.dims || i < y.dims; ++i) {
    const int64_t cx = i < x.dims ? x.count[i] : 1, cy = i < y.dims ? y.count[i] : 1;
    if (cx < 1 || cy < 1) return false;  // no rows
    if (cx > 1 && cy > 1 && x.stride[i] == y.stride[i]) {
      add(x.stride[i], 1 - cy, cx - 1);
    } else {
      if (cx > 1) add(x.stride[i], 0, cx - 1);
      if (cy > 1) add(y.stride[i], 1 - cy, 0);
    }
  }
  wide below = 0, above = 0;
  for (int i = n - 1; i >= 0; --i) {
    t[i].below = below, t[i].above = above;
    below += t[i].lo * t[i].stride, above += t[i].hi * t[i].stride;
  }
  const wide offset = (wide)(uintptr_t)x.at - (wide)(uintptr_t)y.at, least = -(wide)x.bytes, most = y.bytes;  // least < difference < most
  int steps = 4096;
  auto floor_div = [](wide a, wide b) { return a >= 0 ? a / b : -((-a + b - 1) / b); };
  auto search = [&](auto& self, int i, wide v) -> bool {
    if (i == n) return least < v && v < most;
    wide lo = floor_div(least - v - t[i].above, t[i].stride) + 1, hi = -floor_div(-(most - v - t[i].below), t[i].stride) - 1;
    if (lo < t[i].lo) lo = t[i].lo;
    if (hi > t[i].hi) hi = t[i].hi;
    for (wide k = lo; k <= hi; ++k)
      if (--steps < 0 || self(self, i + 1, v + k * t[i].stride)) return steps >= 0;
    return false;
  };
  return search(search, 0, offset);
}

}  // namespace stand
