// Matrix-vector products of MX weights: y[r, n] = sum_j W[n, j] x[r, sigma[j]],
// up to 16 rows of bf16 x that are not quantised, every row against one weight or
// against its expert's.  Bound by the weight stream.
//
// A code times its block's power of two has at most 4 significant bits, so the
// gfx950 scaled conversions give the weight's exact value in bf16 (half an
// instruction per element or less), and the products run on the bf16 MFMA
// 16 x 16 x 32 with fp32 sums: 16 weight rows by up to 16 rows of x.  Which channels
// a lane's 8 values of a product are does not matter as long as both operands
// agree, so a lane takes a packed block whole: lane 16 q + r holds block q of row
// r of a layout step, and product i of the step its elements 8 i .. 8 i + 7.
//
// x is put into that order first, by a launch of its own (16 bytes per lane and
// product then come from L2 in one load); sigma's gather is done once per call
// instead of once per workgroup.
#include "gemm_common.hpp"
#include "gemm_route.hpp"
#include "grouped.hpp"

namespace mm {

namespace {

typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x32v __attribute__((ext_vector_type(32)));
typedef unsigned int u32x6 __attribute__((ext_vector_type(6)));
typedef unsigned int u32x16v __attribute__((ext_vector_type(16)));

constexpr int kWaves = 8, kThreads = 64 * kWaves;

// This lane's block of 32 codes (group G) as bf16 values, two per dword.
template <int G, int FS>
__device__ __forceinline__ u32x16v decode(const v8i& c, float scale) {
  u32x16v v;
  if constexpr (G == 0) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t w = (uint32_t)c[k];
      v[4 * k + 0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
      v[4 * k + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
      v[4 * k + 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
      v[4 * k + 3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
    }
  } else if constexpr (G == 1) {
    const u32x6 w = {(uint32_t)c[0], (uint32_t)c[1], (uint32_t)c[2], (uint32_t)c[3], (uint32_t)c[4], (uint32_t)c[5]};
    if constexpr (FS & 1) v = __builtin_bit_cast(u32x16v, __builtin_amdgcn_cvt_scalef32_pk32_bf16_fp6(w, scale));
    else v = __builtin_bit_cast(u32x16v, __builtin_amdgcn_cvt_scalef32_pk32_bf16_bf6(w, scale));
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t w = (uint32_t)c[k];
      if constexpr (FS & 2) {
        v[2 * k] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, false));
        v[2 * k + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, true));
      } else {
        v[2 * k] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
        v[2 * k + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true));
      }
    }
  }
  return v;
}

// Codes of block q of row n at step s of group G (E4M3: both halves).
template <int G>
__device__ __forceinline__ v8i load_block(const uint8_t* base, int64_t rp, int64_t n, int64_t s, int q) {
  const uint8_t* p = base + code_offset<G>(s, rp, n, q);
  v8i v = {0, 0, 0, 0, 0, 0, 0, 0};
  if constexpr (G == 1) {
    const uint2 a = gload8(p), b = gload8(p + 8), c = gload8(p + 16);
    v[0] = (int)a.x, v[1] = (int)a.y, v[2] = (int)b.x, v[3] = (int)b.y, v[4] = (int)c.x, v[5] = (int)c.y;
  } else {
    const uint4 a = gload16<true>(p);
    v[0] = (int)a.x, v[1] = (int)a.y, v[2] = (int)a.z, v[3] = (int)a.w;
    if constexpr (G == 2) {
      const uint4 b = gload16<true>(p + 512);
      v[4] = (int)b.x, v[5] = (int)b.y, v[6] = (int)b.z, v[7] = (int)b.w;
    }
  }
  return v;
}

// Words of 8 values of x in product order: row `row` of `rows`, global step t,
// product i, block q.
__device__ __forceinline__ int64_t x_word(int rows, int t, int i, int q, int row) {
  return ((int64_t)(t * 16 + i * 4 + q)) * rows + row;
}

// Group G's steps w, w + W, ... of a 32-row tile of the weight.
template <int G, int FS>
__device__ __forceinline__ void gemv_group(const GemvArgs& a, const uint8_t* wq, const uint8_t* wsc, const u32x4* xp,
                                           v4f (&acc)[2], int64_t n0, int row, int wave, int W, int lane) {
  const int S = a.steps[G], q = lane >> 4, r = lane & 15;
  const int t0 = (G >= 1 ? a.steps[0] : 0) + (G >= 2 ? a.steps[1] : 0);
  for (int s = wave; s < S; s += W) {
    u32x4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = xp[x_word(a.rows, t0 + s, i, q, row)];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t n = n0 + 16 * h + r;
      const v8i c = load_block<G>(wq, a.w.rp, n, s, q);
      const float scale = __uint_as_float((uint32_t)load_scale(wsc, a.w.rp, t0 + s, n, q) << 23);
      const u32x16v v = decode<G, FS>(c, scale);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x4 w = {v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
        acc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x[i]),
                                                         acc[h], 0, 0, 0);
      }
    }
  }
}

}  // namespace

// x in product order (x_word), zeros in a group's padding blocks.
__global__ __launch_bounds__(256) void gemv_arrange_kernel(GemvArgs a, u32x4* xp) {
  const int T = a.steps[0] + a.steps[1] + a.steps[2];
  const int64_t words = (int64_t)T * 16 * a.rows;
  const int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (w >= words) return;
  const int row = (int)(w % a.rows), b = (int)(w / a.rows);
  const int q = b & 3, i = (b >> 2) & 3, t = b >> 4;
  const int G = t < a.steps[0] ? 0 : (t < a.steps[0] + a.steps[1] ? 1 : 2);
  const int s = t - (G >= 1 ? a.steps[0] : 0) - (G >= 2 ? a.steps[1] : 0);
  const int blk = 4 * s + q;
  u32x4 v = {0, 0, 0, 0};
  const int e = a.ids ? a.ids[row] : 0;
  if (blk < a.nb[G] && (unsigned)e < (unsigned)a.experts) {
    const int at = 32 * ((G >= 1 ? a.nb[0] : 0) + (G >= 2 ? a.nb[1] : 0) + blk) + 8 * i;
    const int32_t* perm = a.perm + e * a.perm_stride + at;
    const uint16_t* x = a.x + (int64_t)(row / a.top_k) * a.ldx;
    uint32_t u[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int p = perm[k];
      u[k] = x[(unsigned)p < (unsigned)a.K ? p : 0];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = u[2 * k] | u[2 * k + 1] << 16;
  }
  xp[w] = v;
}

// Workgroup (b, u): weight rows 32 b .. of row u's expert, for every row with that
// expert (the first such row's workgroups; without ids, all rows).
template <int FS>
__global__ __launch_bounds__(kThreads) void gemv_kernel(GemvArgs a, const u32x4* xp, int w0, int w1, int w2) {
  __shared__ v4f red[kWaves][2][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q = lane >> 4, c = lane & 15;
  int e = 0, row = c < a.rows ? c : -1;  // this lane's row of x
  if (a.ids) {
    const int u = blockIdx.y;
    e = a.ids[u];
    if ((unsigned)e >= (unsigned)a.experts) return;  // uniform
    const bool same = c < a.rows && a.ids[c < a.rows ? c : 0] == e;
    const uint32_t m = (uint32_t)__ballot(same) & 0xFFFF;
    if ((m & ((1u << u) - 1)) != 0) return;  // uniform: an earlier row's workgroups do it
    row = same ? c : -1;
  }
  const int64_t n0 = (int64_t)blockIdx.x * 32;
  v4f acc[2] = {v4f{0.f, 0.f, 0.f, 0.f}, v4f{0.f, 0.f, 0.f, 0.f}};
  const uint8_t* sc = a.w.sc + e * a.next.sc;
  const int xr = row < 0 ? 0 : row;  // (a column without a row: its results are not stored)
  if (wave < w0) gemv_group<0, FS>(a, a.w.q[0] + e * a.next.q[0], sc, xp, acc, n0, xr, wave, w0, lane);
  else if (wave < w0 + w1) gemv_group<1, FS>(a, a.w.q[1] + e * a.next.q[1], sc, xp, acc, n0, xr, wave - w0, w1, lane);
  else if (wave < w0 + w1 + w2)
    gemv_group<2, FS>(a, a.w.q[2] + e * a.next.q[2], sc, xp, acc, n0, xr, wave - w0 - w1, w2, lane);
  red[wave][0][lane] = acc[0];
  red[wave][1][lane] = acc[1];
  __syncthreads();
  if (wave >= 2 || row < 0) return;
  v4f s = red[0][wave][lane];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) s += red[w][wave][lane];
  const int64_t n = n0 + 16 * wave + 4 * q, N = a.w.rows;
  uint16_t* dst = a.y + (int64_t)row * a.ldy + n;
  if (n + 3 < N) {
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2_rne(s[0], s[1]), pack_bf16x2_rne(s[2], s[3]));
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (n + k < N) dst[k] = (uint16_t)(pack_bf16x2_rne(s[k], 0.f) & 0xFFFF);
  }
}

template <int FS>
static hipError_t launch_gemv_fs(const GemvArgs& a, hipStream_t stream) {
  u32x4* xp = static_cast<u32x4*>(a.workspace);
  const int64_t words = (int64_t)(a.steps[0] + a.steps[1] + a.steps[2]) * 16 * a.rows;
  hipLaunchKernelGGL(gemv_arrange_kernel, dim3((unsigned)((words + 255) / 256)), dim3(256), 0, stream, a, xp);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  int w[3];
  share_waves(a.steps, kEvenCost, kWaves, w);
  hipLaunchKernelGGL((gemv_kernel<FS>), dim3((unsigned)((a.w.rows + 31) / 32), a.ids ? a.rows : 1), dim3(kThreads), 0, stream,
                     a, xp, w[0], w[1], w[2]);
  return hipGetLastError();
}

// The format set is a compile-time choice of conversions: one kernel per set.
hipError_t launch_gemv(const GemvArgs& a, const Device&, hipStream_t stream) {
  switch (a.fs) {
    case 0: return launch_gemv_fs<0>(a, stream);
    case 1: return launch_gemv_fs<1>(a, stream);
    case 2: return launch_gemv_fs<2>(a, stream);
    case 3: return launch_gemv_fs<3>(a, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace mm
