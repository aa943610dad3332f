// Fused gather-by-expert, reorder and quantize: mm_quantize_act's transform of
// the rows that a row-group map puts in each packed row, with the channel order of
// the row's expert.  The codes and scales of a row are those of quantize.hip
// (one block's conversion is shared, quantize_common.hpp); only rows that hold a
// slot are read and written.
//
// HBM-bound: 2 bytes per element in (a token's row is read once per expert that
// takes it, after the first time from the caches), bits / 8 + 1 / 32 out.  A
// workgroup takes a run of consecutive passes of RH packed rows, one thread per
// (row, 32-channel block): the rows go to LDS with 16-byte loads, each thread
// gathers its block by sigma and writes its codes.  sigma stays in registers
// until the expert changes, and a run of passes keeps the rows of a 32-row group,
// which share cache lines in the packed layout, in one L2.
#include "grouped.hpp"
#include "quantize_common.hpp"

namespace mm {

namespace {
constexpr int kMaxQuantThreads = 1024;
}

template <int RH>
__global__ __launch_bounds__(kMaxQuantThreads) void quantize_grouped_kernel(QuantGroupedArgs ga) {
  extern __shared__ __attribute__((aligned(16))) uint8_t stage[];
  const QuantArgs& a = ga.q;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t*)stage;
  const int K = a.K, nblk = K >> 5;
  const int tid = threadIdx.x;
  const int n_act = RH * nblk;
  const bool active = tid < n_act;
  const int t = active ? tid : 0;
  const int blk = t / RH, prow = t - blk * RH;
  const uint32_t row_stride = (uint32_t)(2 * K + 16);

  const int64_t passes = ga.starts[ga.experts] / RH;  // (a multiple of 32 rows)
  const int64_t q_end = passes * (blockIdx.x + 1) / gridDim.x;

  const int group = blk < a.nb[0] ? 0 : (blk < a.nb[0] + a.nb[1] ? 1 : 2);
  const int b = blk - (group >= 1 ? a.nb[0] : 0) - (group >= 2 ? a.nb[1] : 0);
  const int gstep0 = (group >= 1 ? a.steps[0] : 0) + (group >= 2 ? a.steps[1] : 0);
  const bool last = b == (group == 0 ? a.nb[0] : (group == 1 ? a.nb[1] : a.nb[2])) - 1;
  uint8_t* const dst = (group == 0 ? a.q[0] + code_offset<0>(b >> 2, a.rp, prow, b & 3)
                                   : (group == 1 ? a.q[1] + code_offset<1>(b >> 2, a.rp, prow, b & 3)
                                                 : a.q[2] + code_offset<2>(b >> 2, a.rp, prow, b & 3)));
  uint8_t* const sdst = a.sc + ((gstep0 + (b >> 2)) * a.rp + prow) * kStepBlocks + (b & 3);

  constexpr int kParts = 4 / RH;  // a row's 16-byte chunks over the threads: kParts each
  uint32_t sig[16] = {};
  int owner = -1;
  for (int64_t q = passes * blockIdx.x / gridDim.x; q < q_end; ++q) {
    const int64_t row0 = q * RH;
    int32_t slot[RH];
#pragma unroll
    for (int j = 0; j < RH; ++j) slot[j] = ga.slots[row0 + j];
    if (slot[0] < 0) continue;  // uniform: an expert's rows come first in its row groups
    u32x4 buf[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int32_t s = slot[j / kParts] < 0 ? slot[0] : slot[j / kParts];
      const int64_t row = (uint32_t)s / ga.top_k;
      const uint8_t* src = reinterpret_cast<const uint8_t*>(a.x + row * a.ldx + j % kParts * n_act * 8);
      buf[j] = *reinterpret_cast<const u32x4*>(src + (uint32_t)t * 16u);
    }
    const int e = ga.owners[row0 / kRowGroup];
    if (e != owner) {
      owner = e;
      const int32_t* perm = a.perm + e * ga.perm_stride;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int4 v = *reinterpret_cast<const int4*>(perm + blk * 32 + 4 * k);
        const int p[4] = {v.x, v.y, v.z, v.w};
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = 2u * (uint32_t)((unsigned)p[i] < (unsigned)K ? p[i] : 0);
        sig[2 * k] = o[0] | (o[1] << 16);
        sig[2 * k + 1] = o[2] | (o[3] << 16);
      }
    }
    if (active)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        lds_store<u32x4>(lds0 + (uint32_t)(j / kParts) * row_stride + (uint32_t)(j % kParts * n_act + t) * 16u, buf[j]);
    __syncthreads();
    uint32_t base = lds0 + (uint32_t)prow * row_stride;
    asm volatile("" : "+v"(base));  // (see add_word)
    uint32_t d[16];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint16_t v[16];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[2 * i] = lds_u16(add_word<0>(base, sig[8 * h + i]));
        v[2 * i + 1] = lds_u16(add_word<1>(base, sig[8 * h + i]));
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        u16x2 w;
        w.x = v[2 * i];
        w.y = v[2 * i + 1];
        d[8 * h + i] = __builtin_bit_cast(uint32_t, w);
      }
    }
    bool filled = false;
#pragma unroll
    for (int j = 0; j < RH; ++j) filled |= prow == j && slot[j] >= 0;
    if (active && filled) encode_block(d, group, last, a, row0, prow, b, gstep0, dst, sdst);
    __syncthreads();
  }
}

template <int RH>
static hipError_t launch_rows_grouped(const QuantGroupedArgs& a, const Device& dev, hipStream_t stream) {
  static DeviceOnce once;
  constexpr int kLds = 160 * 1024;
  hipError_t e = allow_lds(once, dev, reinterpret_cast<const void*>(quantize_grouped_kernel<RH>), kLds);
  if (e != hipSuccess) return e;
  const int waves = (RH * (a.q.K >> 5) + 63) / 64;
  const size_t lds = (size_t)RH * (2 * a.q.K + 16);
  if (64 * waves > kMaxQuantThreads || lds > kLds) return hipErrorInvalidValue;  // cannot happen: see below
  int64_t per = waves <= 4 ? 16 / waves : 4 / ((waves + 3) / 4);  // (as quantize.hip's launch)
  if (per * lds > kLds) per = kLds / lds;
  const int64_t passes = a.q.rp / RH, cap = per * dev.cus;
  hipLaunchKernelGGL((quantize_grouped_kernel<RH>), dim3((unsigned)(passes < cap ? passes : cap)), dim3(64 * waves), lds,
                     stream, a);
  return hipGetLastError();
}

hipError_t launch_quantize_grouped(const QuantGroupedArgs& a, const Device& dev, hipStream_t stream) {
  const int64_t n = a.q.rp * a.q.K;
  int rh = a.q.K <= 8192 ? 4 : (a.q.K <= 16384 ? 2 : 1);
  if (n < (1 << 20)) rh = 1;
  switch (rh) {
    case 1: return launch_rows_grouped<1>(a, dev, stream);
    case 2: return launch_rows_grouped<2>(a, dev, stream);
    default: return launch_rows_grouped<4>(a, dev, stream);
  }
}

}  // namespace mm
