// Which kernel multiplies rows grouped by expert.  Host arithmetic only, no HIP:
// tests compile it by itself.
//
// The host knows how many slots and experts there are, not how many rows each
// expert has.  Expected tiles of BM rows, with S slots on A = min(experts, S) experts:
// S / BM, and half a tile more for each expert (a whole one where the experts have
// far fewer rows than a tile).
#pragma once

#include "gemm_route.hpp"

namespace mm {

struct GroupedSizes {
  int64_t slots, experts, n;  // n: weight rows of an expert
  int steps[3];
  int cus;
  int64_t ntiles[3];          // tile lists' lengths: 32, 128, 256 rows
};

// Estimates in us: per call, per round of tiles over the CUs (at least one), per
// round and step (kStepTime), per 2^20 bytes of the experts' weights and of the rows
// with their results.  Fitted to 15000 sizes (1 .. 8192 slots, 2 .. 64 experts, K 512 ..
// 14336, N 256 .. 14336, even to very uneven experts) on 256 CUs, weights from HBM,
// within 13-18 % in the mean square: the unevenness, which the host does not know, is
// most of it.  The choice loses 2.8 % to the best kernel in the mean, at worst
// 1.57 times (two experts, one with nearly all of the rows).  With the 32 x 32, 64 x
// 32 and the tiled kernels alone the mean is the same and the worst 1.95 times, K
// 13312 with few weight rows, where 64 x 128 tiles take half as long as the others;
// 64 x 64 tiles change nothing.
struct GroupedCost {
  double once, round, step, w, xy;
};
struct GroupedChoice {
  GemmKernel kernel;
  int shape;       // index into kSplitShapes (kSplit)
  int tn, tm, list, threads;
  GroupedCost cost;
};
constexpr GroupedChoice kGroupedChoices[] = {
    {GemmKernel::kSplit, 0, 1, 1, 0, 512, {3.26, 0, 0.0421, 0.0594, 0.840}},
    {GemmKernel::kSplit, 1, 2, 1, 0, 512, {3.20, 0.243, 0.0494, 0.0849, 0.670}},
    {GemmKernel::kSplit, 4, 2, 4, 1, 512, {3.23, 2.13, 0.0852, 0.0746, 0.903}},
    {GemmKernel::kTiled128, 0, 8, 4, 1, 512, {3.64, 2.57, 0.278, 0.0646, 0.343}},
    {GemmKernel::kTiled256, 0, 8, 8, 2, 256, {5.12, 5.21, 0.459, 0.0592, 0.411}},
};

// shape -1: no kernel's grid takes the sizes.
inline GemmRoute grouped_route(const GroupedSizes& a) {
  constexpr double kMB = 1 << 20;
  constexpr int64_t kMaxThreads = (int64_t)1 << 32;  // a launch has fewer
  const int* S = a.steps;
  const double active = (double)(a.experts < a.slots ? a.experts : a.slots), slots = (double)a.slots;
  const double row_bytes = 68.0 * S[0] + 100.0 * S[1] + 132.0 * S[2];  // with scales
  const int64_t rn = ceil_div(a.n, 32) * 32;
  const double w = active * (double)rn * row_bytes / kMB;
  const double xy = (slots * row_bytes + 2 * slots * (double)a.n) / kMB;
  const double steps = S[0] * kStepTime[0] + S[1] * kStepTime[1] + S[2] * kStepTime[2];
  GemmRoute best = {GemmKernel::kTiled256, -1};
  double least = 0;
  for (const GroupedChoice& c : kGroupedChoices) {
    if (32 * c.tn > rn && c.kernel == GemmKernel::kSplit) continue;  // the weight has not so many rows
    if (ceil_div(a.n, 32 * c.tn) * a.ntiles[c.list] >= kMaxThreads / c.threads) continue;
    const double per = slots / active / (32 * c.tm);  // tiles' worth of rows per expert
    const double tiles = active * (per + 1 - 0.5 * (per < 1 ? per : 1)) * (double)ceil_div(a.n, 32 * c.tn);
    const double rounds = tiles > a.cus ? tiles / a.cus : 1;
    const double t = c.cost.once + rounds * (c.cost.round + c.cost.step * steps) + c.cost.w * w + c.cost.xy * xy;
    if (best.shape < 0 || t < least) {
      least = t;
      best = {c.kernel, c.shape};
    }
  }
  return best;
}

}  // namespace mm
