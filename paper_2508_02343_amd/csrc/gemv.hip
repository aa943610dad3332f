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
// x has to be in that order as well, gathered by sigma.  Few rows (gemv_route.hpp) a
// workgroup takes into LDS as they are (with experts one row), behind its first
// weight loads, and every wavefront gathers the words of a batch of steps for itself.
// More: a launch of its own puts all of x in order in the workspace, from where the
// lanes load their words (L2).
//
// Measured (us, as graph replays; K x N, split 75 / 18.75 / 6.25 % where not said, weights
// from HBM): 1 row, 4096 x 4096 in (2048, 1024, 1024) 5.6 (2.2 TB/s; quantiser and GEMM
// 3.7 + 4.4), 14336 x 4096 10.6 (3.4 TB/s), 4096 x 14336 10.4 (3.4); two experts of 4096 x
// 14336 in E2M1 15.0 (4.2 TB/s); 16 rows with an expert each of 2048 x 1024 7.8 (2.7 TB/s);
// 8 rows, 27648 x 5120 28.9 (3.0 TB/s), where the words of x from L2, as many bytes as the
// weight's, bound it.  Tried: every workgroup putting all of x in order before it begins
// (6.3, 12.7 and 11.3 on the first three), a persistent workgroup with two batches in
// turn (7.8, 18.1: the registers of the second batch leave a SIMD two wavefronts), one
// step at a time (12.4 with the extra launch).
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
__device__ __forceinline__ int x_word(int rows, int t, int i, int q, int row) { return (t * 16 + i * 4 + q) * rows + row; }

// Channel of place `at` (below K) of sigma, clamped (a caller's wrong entry) to
// stay inside the row.
__device__ __forceinline__ int channel(const GemvArgs& a, int p) { return (unsigned)p < (unsigned)a.K ? p : 0; }

// Where a lane's operands of x come from, and where its results go.
struct Column {
  const u32x4* words;   // from the workspace: all rows' words
  const uint16_t* raw;  // from LDS: the unit's rows as they are
  u32x4* mine;          // and this wavefront's words of a batch
  int rows, row;        // rows there, and this lane's
  int out;              // row of y (-1: none)
};

// Steps that a wavefront loads before their products: what 128 registers take (four
// wavefronts per SIMD), two where x's words (64 bytes per lane and step) are loaded
// with them.
template <int G, int TN, bool kLds>
__host__ __device__ constexpr int batch_steps() { return kLds && (G == 0 || TN == 1) ? 4 : 2; }

// Group G's steps wave, wave + W, ... of 16 TN weight rows from n0 on (expert e's).
// Scale words: lane 16 u + r loads row r's four scales at step u of a batch; lane 16 q
// + r takes byte q of the word of lane 16 u + r.  Rows past the weight's are not
// loaded (their products are not stored).  kLds: a batch's words of x are gathered by
// sigma from the rows in LDS by the wavefront that needs them, a word per lane and
// row.  ready(): called once, behind the first loads, before x is read.
template <int G, int FS, int TN, bool kLds, class Ready>
__device__ __forceinline__ void gemv_group(const GemvArgs& a, int64_t e, const Column& x, v4f (&acc)[TN], int64_t n0, int wave,
                                           int W, int lane, const Ready& ready) {
  constexpr int U = batch_steps<G, TN, kLds>();
  static_assert(U <= 4, "one scale word, and one word of x, per lane for four steps");
  const int q = lane >> 4, r = lane & 15, S = a.steps[G];
  const int t0 = (G >= 1 ? a.steps[0] : 0) + (G >= 2 ? a.steps[1] : 0);
  const uint8_t* wq = a.w.q[G] + e * a.next.q[G];
  const uint8_t* wsc = a.w.sc + e * a.next.sc;
  // kLds: lane 16 u + 4 i + k gathers word (i, k) of step u
  const int32_t* perm = a.perm + e * a.perm_stride + 32 * ((G >= 1 ? a.nb[0] : 0) + (G >= 2 ? a.nb[1] : 0));
  const int gi = (lane >> 2) & 3, gk = lane & 3;
  bool first = true;
  for (int s0 = wave; s0 < S || first; s0 += W * U) {
    int4 plo = {0, 0, 0, 0}, phi = plo;
    bool gather = false;  // this lane's word is not padding
    if constexpr (kLds) {
      const int blk = 4 * (s0 + W * q) + gk;
      gather = q < U && blk < a.nb[G];
      if (gather) {
        const int4* p = reinterpret_cast<const int4*>(perm + 32 * blk + 8 * gi);
        plo = p[0];
        phi = p[1];
      }
    }
    v8i w[U][TN];
    uint32_t sw[TN];
    const int su = s0 + W * q;
#pragma unroll
    for (int i = 0; i < TN; ++i)
      sw[i] = q < U && su < S && n0 + 16 * i + r < a.w.rows
                  ? *(const __attribute__((address_space(1))) uint32_t*)(wsc + ((t0 + su) * a.w.rp + n0 + 16 * i + r) * kStepBlocks)
                  : 0u;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + W * u;
      if (s < S)  // uniform
#pragma unroll
        for (int i = 0; i < TN; ++i)
          if (n0 + 16 * i + r < a.w.rows) w[u][i] = load_block<G>(wq, a.w.rp, n0 + 16 * i + r, s, q);
    }
    u32x4 xv[kLds ? 1 : U][4];
    if constexpr (!kLds)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int s = s0 + W * u;
        if (s < S && x.out >= 0)
#pragma unroll
          for (int i = 0; i < 4; ++i) xv[u][i] = x.words[x_word(x.rows, t0 + s, i, q, x.row)];
      }
    __builtin_amdgcn_sched_barrier(0);  // all of the batch's loads go out before its first product
    if (first) ready();
    first = false;
    if constexpr (kLds) {
      if (q < U) {
        const int ch[8] = {plo.x, plo.y, plo.z, plo.w, phi.x, phi.y, phi.z, phi.w};
        for (int k = 0; k < x.rows; ++k) {
          const uint16_t* row = x.raw + k * a.K;
          u32x4 v;
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = row[channel(a, ch[2 * j])] | (uint32_t)row[channel(a, ch[2 * j + 1])] << 16;
          x.mine[lane * x.rows + k] = gather ? v : u32x4{0, 0, 0, 0};
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + W * u;
      if (s >= S) break;  // uniform
      if constexpr (kLds)
#pragma unroll
        for (int i = 0; i < 4; ++i) xv[0][i] = x.mine[(16 * u + 4 * i + q) * x.rows + x.row];
#pragma unroll
      for (int h = 0; h < TN; ++h) {
        const uint32_t word = (uint32_t)__builtin_amdgcn_ds_bpermute((16 * u + r) * 4, (int)sw[h]);
        const u32x16v v = decode<G, FS>(w[u][h], __uint_as_float((word >> (8 * q) & 0xFF) << 23));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const u32x4 k = {v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
          acc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k),
                                                           __builtin_bit_cast(bf16x8, xv[kLds ? 0 : u][i]), acc[h], 0, 0, 0);
        }
      }
    }
    if constexpr (kLds) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// Four columns n .. n + 3 of row `row` of y.
__device__ __forceinline__ void store_four(const GemvArgs& a, int64_t row, int64_t n, const v4f& s) {
  const int64_t N = a.w.rows;
  uint16_t* dst = a.y + row * a.ldy + n;
  if (n + 3 < N) {
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2_rne(s[0], s[1]), pack_bf16x2_rne(s[2], s[3]));
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (n + k < N) dst[k] = (uint16_t)(pack_bf16x2_rne(s[k], 0.f) & 0xFFFF);
  }
}

// The place in sigma of word (t, i, q) of x, or -1 in a group's padding.
__device__ __forceinline__ int place_of(const GemvArgs& a, int b) {
  const int q = b & 3, i = (b >> 2) & 3, t = b >> 4;
  const int G = t < a.steps[0] ? 0 : (t < a.steps[0] + a.steps[1] ? 1 : 2);
  const int s = t - (G >= 1 ? a.steps[0] : 0) - (G >= 2 ? a.steps[1] : 0);
  const int blk = 4 * s + q;
  if (blk >= (G == 0 ? a.nb[0] : (G == 1 ? a.nb[1] : a.nb[2]))) return -1;
  return 32 * ((G >= 1 ? a.nb[0] : 0) + (G >= 2 ? a.nb[1] : 0) + blk) + 8 * i;
}

}  // namespace

// x in product order (x_word), zeros in a group's padding blocks.
__global__ __launch_bounds__(256) void gemv_arrange_kernel(GemvArgs a, u32x4* xp) {
  const int words = (a.steps[0] + a.steps[1] + a.steps[2]) * 16 * a.rows;
  const int w = (int)blockIdx.x * 256 + threadIdx.x;
  if (w >= words) return;
  const int row = w % a.rows, at = place_of(a, w / a.rows);
  u32x4 v = {0, 0, 0, 0};
  const int e = a.ids ? a.ids[row] : 0;
  if (at >= 0 && (unsigned)e < (unsigned)a.experts) {
    const int4* perm = reinterpret_cast<const int4*>(a.perm + e * a.perm_stride + at);
    const int4 lo = perm[0], hi = perm[1];
    const int p[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    const uint16_t* x = a.x + (int64_t)(row / a.top_k) * a.ldx;
    uint32_t u[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) u[k] = x[channel(a, p[k])];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = u[2 * k] | u[2 * k + 1] << 16;
  }
  xp[w] = v;
}

// Workgroup (b, u): weight rows 16 TN b .. of unit u's weight.  A unit is a row's
// expert, or without ids the one weight for all rows.  kLds: the unit's rows of x
// are put into LDS as they are (dynamic; behind them each wavefront's words); with
// ids one row, so that every row is a unit of its own.  Else x comes from the
// workspace, where an earlier launch put it in order, and the first row with an
// expert is the unit for all rows with it (columns of one product).
template <int FS, int TN, int kWaves, bool kLds>
__global__ __launch_bounds__(64 * kWaves, 4) void gemv_kernel(GemvArgs a, const u32x4* xp, int w0, int w1, int w2) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  __shared__ v4f red[kWaves][TN][64];
  const int lane = threadIdx.x & 63, tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q = lane >> 4, c = lane & 15;
  const int unit = blockIdx.y;
  const int e = a.ids ? a.ids[unit] : 0;
  if ((unsigned)e >= (unsigned)a.experts) return;  // uniform
  const int rows = kLds && a.ids ? 1 : a.rows;
  Column x;
  x.words = xp;
  x.raw = reinterpret_cast<const uint16_t*>(lds);
  x.mine = reinterpret_cast<u32x4*>(lds + (size_t)rows * a.K * 2) + wave * 64 * rows;
  x.rows = rows;
  x.row = c < rows ? c : 0;
  x.out = c < rows ? c : -1;
  if (a.ids) {
    if constexpr (kLds) {
      x.out = c == 0 ? unit : -1;
    } else {
      const bool same = c < a.rows && a.ids[c < a.rows ? c : 0] == e;
      const uint32_t m = (uint32_t)__ballot(same) & 0xFFFF;
      if ((m & ((1u << unit) - 1)) != 0) return;  // uniform: an earlier unit's
      x.out = same ? c : -1;
    }
  }
  auto ready = [&] {
    if constexpr (!kLds) return;
    const int chunks = a.K >> 3;  // 16-byte chunks per row
    const bool wide = (((uintptr_t)a.x | (uintptr_t)(a.ldx * 2)) & 15) == 0;
    for (int r = 0; r < rows; ++r) {
      const uint16_t* src = a.x + (int64_t)((a.ids ? unit : r) / a.top_k) * a.ldx;
      for (int k = tid; k < chunks; k += 64 * kWaves) {
        u32x4 v;
        if (wide) {
          v = *reinterpret_cast<const u32x4*>(src + 8 * k);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = src[8 * k + 2 * j] | (uint32_t)src[8 * k + 2 * j + 1] << 16;
        }
        *reinterpret_cast<u32x4*>(lds + (size_t)r * a.K * 2 + 16 * k) = v;
      }
    }
    __syncthreads();
  };
  const int64_t n0 = (int64_t)blockIdx.x * (16 * TN);
  v4f acc[TN];
#pragma unroll
  for (int i = 0; i < TN; ++i) acc[i] = v4f{0.f, 0.f, 0.f, 0.f};
  if (wave < w0) gemv_group<0, FS, TN, kLds>(a, e, x, acc, n0, wave, w0, lane, ready);
  else if (wave < w0 + w1) gemv_group<1, FS, TN, kLds>(a, e, x, acc, n0, wave - w0, w1, lane, ready);
  else gemv_group<2, FS, TN, kLds>(a, e, x, acc, n0, wave - w0 - w1, w2, lane, ready);
#pragma unroll
  for (int i = 0; i < TN; ++i) red[wave][i][lane] = acc[i];
  __syncthreads();
  if (wave >= TN || x.out < 0) return;
  v4f s = red[0][wave][lane];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) s += red[w][wave][lane];
  store_four(a, x.out, n0 + 16 * wave + 4 * q, s);
}

// What a launch is asked: the plan is the rule's (gemv_route.hpp).
static GemvSizes sizes_of(const GemvArgs& a, const Device& dev) {
  return GemvSizes{a.rows, a.K, a.w.rows, a.ids ? a.experts : 0, dev.cus};
}

template <int FS, int TN, int W>
static hipError_t launch_gemv_strip(const GemvArgs& a, bool in_lds, const Device& dev, hipStream_t stream) {
  int w[3];
  share_waves(a.steps, kByteCost, W, w);
  const dim3 grid((unsigned)((a.w.rows + 16 * TN - 1) / (16 * TN)), a.ids ? a.rows : 1);
  if (in_lds) {
    static DeviceOnce once;
    hipError_t e = allow_lds(once, dev, reinterpret_cast<const void*>(gemv_kernel<FS, TN, W, true>), (int)kGemvMaxLds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((gemv_kernel<FS, TN, W, true>), grid, dim3(64 * W), (size_t)gemv_lds_bytes(a.ids ? 1 : a.rows, a.K, W),
                       stream, a, nullptr, w[0], w[1], w[2]);
    return hipGetLastError();
  }
  u32x4* xp = static_cast<u32x4*>(a.workspace);
  const int64_t words = (int64_t)(a.steps[0] + a.steps[1] + a.steps[2]) * 16 * a.rows;
  hipLaunchKernelGGL(gemv_arrange_kernel, dim3((unsigned)((words + 255) / 256)), dim3(256), 0, stream, a, xp);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((gemv_kernel<FS, TN, W, false>), grid, dim3(64 * W), 0, stream, a, xp, w[0], w[1], w[2]);
  return hipGetLastError();
}

template <int FS>
static hipError_t launch_gemv_fs(const GemvArgs& a, const Device& dev, hipStream_t stream) {
  const GemvPlan p = gemv_plan(sizes_of(a, dev));
  if (p.tn == 1) return launch_gemv_strip<FS, 1, 16>(a, p.in_lds, dev, stream);
  switch (p.waves) {
    case 16: return launch_gemv_strip<FS, 2, 16>(a, p.in_lds, dev, stream);
    case 8: return launch_gemv_strip<FS, 2, 8>(a, p.in_lds, dev, stream);
    default: return launch_gemv_strip<FS, 2, 4>(a, p.in_lds, dev, stream);
  }
}

// The format set is a compile-time choice of conversions: one kernel per set.
hipError_t launch_gemv(const GemvArgs& a, const Device& dev, hipStream_t stream) {
  switch (a.fs) {
    case 0: return launch_gemv_fs<0>(a, dev, stream);
    case 1: return launch_gemv_fs<1>(a, dev, stream);
    case 2: return launch_gemv_fs<2>(a, dev, stream);
    case 3: return launch_gemv_fs<3>(a, dev, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace mm
