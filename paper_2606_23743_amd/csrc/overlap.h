// Whether two strided tensors share a byte.  Host only, no HIP.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace sva {

// Rows of `row` bytes from `at` on, in up to three dimensions (sizes >= 1, strides in bytes >= 0).
struct RowSet {
  uint64_t at;
  int64_t row;
  int64_t size[3], stride[3];
};

// The multiples of one stride that rows of x may lie behind rows of y by, and what it and the
// shorter strides add at least and at most.
struct RowSteps {
  int64_t stride, first, last;
  int64_t lo, hi;
};

// Whether `at` and a sum of steps falls between `below` and `above`: the longest stride first,
// and only by as many steps as the shorter ones can make up for.  Layouts too entangled for
// `budget` of them count as if.
inline bool steps_reach(const RowSteps* d, int n, int64_t at, int64_t below, int64_t above, int* budget) {
  if (--*budget < 0) return true;
  if (n == 0) return at > below && at < above;
  const int64_t lo = n > 1 ? d[1].lo : 0, hi = n > 1 ? d[1].hi : 0, s = d->stride;
  auto down = [](int64_t a, int64_t b) { return a / b - (a % b != 0 && a < 0); };
  const int64_t first = std::max(d->first, down(below - hi - at, s) + 1);
  const int64_t last = std::min(d->last, -down(at + lo - above, s) - 1);
  for (int64_t k = first; k <= last; ++k)
    if (steps_reach(d + 1, n - 1, at + k * s, below, above, budget)) return true;
  return false;
}

// Rows that interleave without touching (slices of one projection) share nothing.
inline bool rows_meet(const RowSet& x, const RowSet& y) {
  RowSteps d[6];
  int n = 0;
  auto add = [&](int64_t size, int64_t stride, bool of_x) {
    if (size == 1 || stride == 0) return;
    int i = 0;
    while (i < n && d[i].stride != stride) ++i;
    if (i == n) d[n++] = {stride, 0, 0, 0, 0};
    if (of_x) d[i].last += size - 1;
    else d[i].first -= size - 1;
  };
  for (int i = 0; i < 3; ++i) {
    add(x.size[i], x.stride[i], true);
    add(y.size[i], y.stride[i], false);
  }
  std::sort(d, d + n, [](const RowSteps& a, const RowSteps& b) { return a.stride > b.stride; });
  for (int i = n - 1; i >= 0; --i) {
    d[i].lo = d[i].first * d[i].stride + (i + 1 < n ? d[i + 1].lo : 0);
    d[i].hi = d[i].last * d[i].stride + (i + 1 < n ? d[i + 1].hi : 0);
  }
  int budget = 4096;
  return steps_reach(d, n, (int64_t)(x.at - y.at), -x.row, y.row, &budget);
}

}  // namespace sva
