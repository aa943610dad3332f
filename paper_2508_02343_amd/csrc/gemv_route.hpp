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

// From LDS (one launch) go rows that fit it with the most wavefronts, and rows that each
// have an expert of their own to find (at least as many experts as rows: a workgroup
// then holds one row).  The others from the workspace, where a launch in front puts
// them in order.  (With experts LDS holds one row; rows that must share experts, as there
// are fewer, share their weights' loads only from the workspace.)
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
