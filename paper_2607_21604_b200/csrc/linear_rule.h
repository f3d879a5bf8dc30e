// How many ranges of columns a linear layer on tcgen05 is cut into; a range is a CTA, and those of the same features and
// rows are a cluster.  Plain C++.
#pragma once
#include <stdint.h>

constexpr int LQ_MAX_RANGES = 8;

// `units` clusters of `pairs` pairs of groups; fit[k], k = 1 .. 8: how many clusters of k CTAs run at a time, 0 where none
// does (a part of the GPU may not hold one).  As many ranges, of four pairs or more each, as give the shortest run: rounds
// of clusters times steps, with 20 for start and end.  0: not even one CTA runs.
inline int lq_ranges(int64_t units, int pairs, const int* fit) {
  int ranges = 0;
  double best = 0;
  for (int k = 1; k <= LQ_MAX_RANGES && (k == 1 || pairs / k >= 4); ++k) {
    if (fit[k] < 1) continue;
    const double cost = (double)((units + fit[k] - 1) / fit[k]) * (2 * ((pairs + k - 1) / k) + 20);
    if (ranges == 0 || cost < best) { best = cost; ranges = k; }
  }
  return ranges;
}
