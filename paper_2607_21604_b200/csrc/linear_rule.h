// How a linear layer's columns are cut into ranges, and which of two kernels takes up to 16 rows.  A range is a CTA, and those of
// the same features and rows are a cluster.  Plain C++.
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

// Clusters that run at a time on a whole B200, by their CTAs (cudaOccupancyMaxActiveClusters): of the kernel on mma.sync, of which
// an SM holds two (float rows: one) and which has 1, 2, 4 or 8 ranges; and of the one on tcgen05, one CTA an SM.
constexpr int LQ_FIT_TWO[9] = {0, 296, 148, 93, 71, 56, 45, 37, 33}, LQ_FIT_ONE[9] = {0, 148, 74, 45, 33, 26, 22, 15, 15};

// Ranges of the kernel on mma.sync, of 512 columns or more each: as many as let every cluster run at once.
inline int lq_cluster_ranges(int64_t units, int groups, const int* fit) {
  int ranges = 1;
  while (ranges < 8 && units <= fit[ranges * 2] && (groups + ranges * 2 - 1) / (ranges * 2) >= 8) ranges *= 2;
  return ranges;
}

// Whether tcgen05 is faster for up to 16 rows of a 16-bit type, by what either kernel takes, in us: 4 and 0.41 a group (0.29 up to
// 8 rows) for every round of clusters, and 2 and 0.33 of the cost above.  Measured, 9 to 16 rows, on mma.sync against tcgen05:
// 4096 x 14336 17.4 / 21.3, 14336 x 4096 17.3 / 18.4, 8192 x 8192 17.5 / 19.0, 4096 x 27648 27.5 / 32.4; 10240 x 8192 31.0 / 23.1,
// 5120 x 14336 27.2 / 21.8, 28672 x 4096 30.6 / 28.3, 20480 x 14336 95.8 / 63.7.  Over 200 sizes the choice is 0.2 % slower than the
// better one in the mean and 10 % at worst (one bound on the size of the weights: 4 % and 48 %).  The estimates go by groups as they
// are, not by whole steps, so that a layer with more columns never changes back.
inline bool lq_prefers_tensor(int rows, int features, int groups) {
  const int64_t units = ((int64_t)features + 127) / 128, wide = ((int64_t)features + 255) / 256;
  const int ranges = lq_cluster_ranges(units, groups, LQ_FIT_TWO), fit = LQ_FIT_TWO[ranges];
  const double mma = (double)((units + fit - 1) / fit) * (4 + (rows <= 8 ? 0.29 : 0.41) * groups / ranges);
  double cost = 0;
  for (int k = 1; k <= LQ_MAX_RANGES && (k == 1 || groups >= 8 * k); ++k) {
    const double c = (double)((wide + LQ_FIT_ONE[k] - 1) / LQ_FIT_ONE[k]) * ((double)groups / k + 20);
    if (k == 1 || c < cost) cost = c;
  }
  return 2 + 0.33 * cost < mma;
}
