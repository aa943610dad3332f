// Which kernel multiplies rows grouped by expert.  Host arithmetic only, no HIP:
// tests compile it by itself.
//
// The host knows how many slots and experts there are, not how many rows each
// expert has.  Expected tiles of BM rows, with S slots on A = min(experts, S) experts:
// S / BM and half a tile more for each expert, at least one each.
#pragma once

#include "gemm_route.hpp"

namespace mm {

// By tile, weight rows x rows: the K-splitting kernel, the LDS-tiled one (Rest: with a last
// round that is at most half full in quarters of a tile).
enum class GroupedKernel { kSplit32x32, kSplit64x32, kTiled128x128, kTiled256x128, kTiled256x256, kTiled256x256Rest, kNone };

struct GroupedSizes {
  int64_t slots, experts, n;  // n: weight rows of an expert
  int steps[3];
  int cus;
  int64_t ntiles[3];          // tile lists' lengths: 32, 128, 256 rows
};

// Estimates in us: per call, per round of tiles over the CUs (at least one; half of a
// round that is not full counts), per round and step (kStepTime), per 2^20 bytes of
// the experts' weights and of the rows with their results.  Fitted to 12500 sizes (1
// .. 8192 slots, 2 .. 64 experts, K 512 .. 14336, N 256 .. 14336, even to very uneven
// experts) on 256 CUs, weights from HBM, within 12-18 % in the mean square: the
// unevenness, which the host does not know, is most of it.  The choice loses 2.6 % to
// the best kernel in the mean, more than 10 % at one size in eleven, at worst 1.7
// times (a few experts with K above 8000 and few weight rows).  Without the 128 x
// 128 tiles (two workgroups on a CU) it lost 3.8 %, at worst 1.8 times; 64 x 64 and 64 x
// 128 tiles of the K-splitting kernel change nothing in the mean.  With the Rest the rounds
// are as many as there are tiles for, and its launch 3 us: over another 15100 sizes 2.1 %
// lost against 2.2 % without it, over those of 80 us or more 2.9 % against 4.9 %.
struct GroupedCost {
  double once, round, step, w, xy;
};
struct GroupedChoice {
  GroupedKernel kernel;
  int tn, tm;         // tile in 32-row units of weight rows and rows
  int list, threads;  // tile list, threads of a workgroup
  GroupedCost cost;
};
constexpr GroupedChoice kGroupedChoices[] = {
    {GroupedKernel::kSplit32x32, 1, 1, 0, 512, {3.37, 0.0881, 0.0379, 0.0649, 0.876}},
    {GroupedKernel::kSplit64x32, 2, 1, 0, 512, {3.31, 0.332, 0.0472, 0.0852, 0.650}},
    {GroupedKernel::kTiled128x128, 4, 4, 1, 256, {5.78, 0.250, 0.209, 0.0424, 0.238}},
    {GroupedKernel::kTiled256x128, 8, 4, 1, 512, {4.38, 2.07, 0.276, 0.0596, 0.278}},
    {GroupedKernel::kTiled256x256, 8, 8, 2, 256, {6.06, 3.30, 0.467, 0.0440, 0.334}},
    {GroupedKernel::kTiled256x256Rest, 8, 8, 2, 256, {9.06, 3.30, 0.467, 0.0440, 0.334}},
};

// kNone: no kernel's grid takes the sizes.
inline GroupedKernel grouped_route(const GroupedSizes& a) {
  constexpr double kMB = 1 << 20;
  constexpr int64_t kMaxThreads = (int64_t)1 << 32;  // a launch has fewer
  const int* S = a.steps;
  const double active = (double)(a.experts < a.slots ? a.experts : a.slots), slots = (double)a.slots;
  const double row_bytes = 68.0 * S[0] + 100.0 * S[1] + 132.0 * S[2];  // with scales
  const int64_t rn = ceil_div(a.n, 32) * 32;
  const double w = active * (double)rn * row_bytes / kMB;
  const double xy = (slots * row_bytes + 2 * slots * (double)a.n) / kMB;
  const double steps = S[0] * kStepTime[0] + S[1] * kStepTime[1] + S[2] * kStepTime[2];
  GroupedKernel best = GroupedKernel::kNone;
  double least = 0;
  for (const GroupedChoice& c : kGroupedChoices) {
    if (c.kernel == GroupedKernel::kSplit64x32 && rn < 64) continue;  // the weight has not so many rows
    const int64_t tiles_n = ceil_div(a.n, 32 * c.tn);
    if (tiles_n * a.ntiles[c.list] >= kMaxThreads / c.threads) continue;
    const double per = slots / active / (32 * c.tm) + 0.5;
    const double q = active * (per > 1 ? per : 1) * (double)tiles_n / a.cus;
    const double up = (double)(int64_t)q < q ? (double)((int64_t)q + 1) : q;
    double rounds = ((q > 1 ? q : 1) + up) / 2;
    if (c.kernel == GroupedKernel::kTiled256x256Rest) rounds = q > 0.65 ? q : 0.65;
    const double t = c.cost.once + rounds * (c.cost.round + c.cost.step * steps) + c.cost.w * w + c.cost.xy * xy;
    if (best == GroupedKernel::kNone || t < least) {
      least = t;
      best = c.kernel;
    }
  }
  return best;
}

}  // namespace mm
