// Which form of the matrix-vector kernel a call takes, and the workspace that it needs.
// Host arithmetic only, no HIP: tests compile it by itself.
#pragma once

#include <stdint.h>

namespace mm {

// At most this many rows in a call of the matrix-vector kernel.
constexpr int kGemvMaxRows = 16;
constexpr int64_t kGemvMaxN = (int64_t)1 << 28;  // (a launch has fewer than 2^32 threads)
constexpr int64_t kGemvMaxK = 32768;

// LDS of a workgroup of `waves` wavefronts that holds `rows` rows of x: the rows, and
// 64 words of each per wavefront; beside it the workgroup has 32 KB of sums.
constexpr int kGemvMaxWaves = 16;
constexpr int64_t kGemvMaxLds = 110 * 1024;
constexpr int64_t gemv_lds_bytes(int64_t rows, int64_t K, int waves) { return rows * (2 * K + 1024 * (int64_t)waves); }
static_assert(gemv_lds_bytes(1, kGemvMaxK, kGemvMaxWaves) <= kGemvMaxLds, "one row fits whatever its length");

struct GemvSizes {
  int64_t rows, K, n;  // n: weight rows of an expert
  int64_t experts;     // 0: one weight for every row, no ids
  int cus;
};

// With experts a workgroup's LDS holds one row, so every row loads its expert's weight for
// itself; from the workspace, where a launch in front puts x in order, rows that share an
// expert are columns of one product and share its loads.  Without ids all rows share the
// one weight either way.  From LDS (one launch) go rows few enough to fit it all together,
// and rows with at least as many experts as rows; the others from the workspace.
//
// Measured with experts chosen at random (us, LDS / workspace; 75 / 18.75 / 6.25 %, weights
// from HBM), where the rule takes LDS: 2 rows on 2 experts of 2048 x 4096 (K x N) 5.5 / 8.3, on 8
// of 4096 x 14336 17.2 / 21.0; 4 rows on 64 experts of 4096 x 4096 12.1 / 14.6; 16 on 64 of 2048
// x 1024 8.2 / 12.1, of 4096 x 14336 90.8 / 95.9; 8 on 8 of 4096 x 4096 16.2 / 19.2, of 4096 x 14336
// 46.3 / 43.1; few rows that fit on fewer experts: 4 on 2 of 2048 x 1024 4.7 / 7.2, of 4096 x 4096
// 9.9 / 10.7, but of 4096 x 14336 26.0 / 19.4.  Where it takes the workspace: 16 rows on 2 of 4096
// x 14336 81.9 / 24.3, on 8 of 4096 x 4096 28.0 / 24.0, 8 on 2 of 14336 x 4096 39.2 / 32.0, but
// small weights stay in the caches and the second launch is not worth it: 16 on 8 of 2048 x
// 1024 6.6 / 10.4, 8 on 2 of 4096 x 4096 13.2 / 13.6.  Over 336 such sizes the choice takes 6 % more
// than the better one in the mean, 1.76 times at worst; LDS only up to as many rows as experts
// would take 10 %, LDS always 10 % and 5.1 times at worst, the workspace always 23 %.
inline bool gemv_in_lds(const GemvSizes& a) {
  return gemv_lds_bytes(a.rows, a.K, kGemvMaxWaves) <= kGemvMaxLds || (a.experts > 0 && a.rows <= a.experts);
}

inline int64_t gemv_workspace_bytes(const GemvSizes& a, const int* steps) {
  return gemv_in_lds(a) ? 0 : a.rows * 256 * ((int64_t)steps[0] + steps[1] + steps[2]);
}

// Strips of 16 tn weight rows, the wavefronts of a strip's workgroup, and where x comes from.
//
// One strip of 16 rows and sixteen wavefronts for every CU as long as there are no more of
// them (us, 1 row, K x N: 4096 x 4096 5.6 against 6.3 with eight and 6.4 with 32 rows, 14336
// x 4096 10.9 / 12.4 / 13.6); above, strips of 32 rows (whole records of the layout), with
// fewer wavefronts the more strips share a CU: four beyond two strips per CU (two experts of
// 14336 x 4096 in E2M1 14.4, with eight 16.3), eight beyond one (14336 rows of K 4096 10.5,
// with four 11.1, with sixteen 11.9), else sixteen (two experts of 4096 x 14336 16.8, with
// eight 18.7).
struct GemvPlan {
  int tn, waves;
  bool in_lds;
};
inline GemvPlan gemv_plan(const GemvSizes& a) {
  const int64_t units = a.experts > 0 ? a.rows : 1, strips = units * ((a.n + 31) / 32);
  const bool in_lds = gemv_in_lds(a);
  if (units * ((a.n + 15) / 16) <= a.cus) return {1, 16, in_lds};
  if (strips <= a.cus) return {2, 16, in_lds};
  if (strips <= 2 * (int64_t)a.cus) return {2, 8, in_lds};
  return {2, 4, in_lds};
}

}  // namespace mm
