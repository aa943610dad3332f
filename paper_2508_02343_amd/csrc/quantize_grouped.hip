// Fused gather-by-expert, reorder and quantize: mm_quantize_act's transform of
// the rows that a row-group map puts in each packed row, with the channel order of
// the row's expert.  The codes and scales of a row are those of quantize.hip
// (one block's conversion is shared, quantize_common.hpp); only rows that hold a
// slot are read and written.
//
// HBM-bound: 2 bytes per element in (a token's row is read once per expert that
// takes it, after the first time from the caches), bits / 8 + 1 / 32 out.  As in
// quantize.hip a workgroup stages a pass of RH packed rows in LDS, one thread per (row,
// 32-channel block), the next pass's rows in flight while it quantises this one, and
// the passes that run together on an XCD are neighbours, so that the rows of a 32-row
// group, which share cache lines in the packed layout, meet in one L2.  sigma stays
// in registers until the expert changes.
//
// Measured (us, as graph replays): 16 rows of K 4096 4.3; 4096 slots x 4096, two per
// token, 14.7 (3.0 TB/s of rows and codes); 8192 slots x 14336, a sigma per expert, 76 (4.0
// TB/s).  A run of consecutive passes to each workgroup took 109 on the last (the lines
// of half-filled row groups do not last in the L2), without the next pass's loads in
// flight 111.
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

  // this workgroup's passes: those of quantize.hip (each XCD a contiguous range, its
  // workgroups in turn), as far as they have rows
  constexpr int kPasses = kRowGroup / RH;  // per row group
  const int64_t used = ga.starts[ga.experts];  // (a multiple of 32 rows)
  const int64_t passes = (used < a.rp ? used : a.rp) / RH;
  int64_t q, q_end, stride;
  if (gridDim.x % 8 == 0) {
    const int x = blockIdx.x & 7;
    q = passes * x / 8 + (blockIdx.x >> 3);
    q_end = passes * (x + 1) / 8;
    stride = gridDim.x / 8;
  } else {
    q = blockIdx.x;
    q_end = passes;
    stride = gridDim.x;
  }
  // Moves q on to a pass with rows, and its row group's tile; an expert's rows come
  // first in its row groups.
  TileRows tile = {};
  auto seek = [&] {  // uniform over the workgroup
    for (; q < q_end; q += stride) {
      tile = tile_rows(ga.tiles[q / kPasses], kRowGroup, a.rp, ga.experts);
      if ((int)(q % kPasses) * RH < tile.rows) return;
    }
  };
  constexpr int kParts = 4 / RH;  // a row's 16-byte chunks over the threads: kParts each
  u32x4 buf[4];
  auto load = [&] {
#pragma unroll
    for (int j = 0; j < RH; ++j) {
      uint32_t s = (uint32_t)ga.slots[q * RH + j];
      if (s >= ga.rows) s = (uint32_t)ga.slots[q * RH];  // (rows without a slot: the pass's first again)
      const int64_t row = (s < ga.rows ? s : 0) / ga.top_k;
#pragma unroll
      for (int k = 0; k < kParts; ++k) {
        const uint8_t* src = reinterpret_cast<const uint8_t*>(a.x + row * a.ldx + k * n_act * 8);
        buf[j * kParts + k] = *reinterpret_cast<const u32x4*>(src + (uint32_t)t * 16u);
      }
    }
  };
  seek();
  if (q >= q_end) return;
  load();

  const int group = blk < a.nb[0] ? 0 : (blk < a.nb[0] + a.nb[1] ? 1 : 2);
  const int b = blk - (group >= 1 ? a.nb[0] : 0) - (group >= 2 ? a.nb[1] : 0);
  const int gstep0 = (group >= 1 ? a.steps[0] : 0) + (group >= 2 ? a.steps[1] : 0);
  const bool last = b == (group == 0 ? a.nb[0] : (group == 1 ? a.nb[1] : a.nb[2])) - 1;
  uint8_t* const dst = (group == 0 ? a.q[0] + code_offset<0>(b >> 2, a.rp, prow, b & 3)
                                   : (group == 1 ? a.q[1] + code_offset<1>(b >> 2, a.rp, prow, b & 3)
                                                 : a.q[2] + code_offset<2>(b >> 2, a.rp, prow, b & 3)));
  uint8_t* const sdst = a.sc + ((gstep0 + (b >> 2)) * a.rp + prow) * kStepBlocks + (b & 3);

  uint32_t sig[16] = {};
  int owner = -1;
  while (q < q_end) {
    const int64_t row0 = q * RH;
    const int e = tile.expert;
    const bool filled = (int)(q % kPasses) * RH + prow < tile.rows;
    if (active)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        lds_store<u32x4>(lds0 + (uint32_t)(j / kParts) * row_stride + (uint32_t)(j % kParts * n_act + t) * 16u, buf[j]);
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
    __syncthreads();
    q += stride;
    seek();
    if (q < q_end) load();  // in flight while this pass is quantised
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

// Rows per pass: two, for the longer runs of codes per store; one above 16384
// channels (1024 threads), and above 8192 as long as every row is in flight at once (128
// x 14336 6.2 / 7.1 us with one / two); four up to 2048 channels unless there is little
// to do (us, 1 / 2 / 4 rows per pass, slots x K: 32 x 1024 4.4 / 4.3 / 4.5, 256 x 1024
// 4.9 / 4.4 / 4.7, 1024 x 1024 6.0 / 5.4 / 4.9, 8192 x 2048 18.0 / 14.8 / 13.7, 1024 x
// 4096 7.4 / 6.6 / 7.4, 8192 x 4096 27.5 / 22.4 / 22.0, 8192 x 8192 52 / 46 / 45).
hipError_t launch_quantize_grouped(const QuantGroupedArgs& a, const Device& dev, hipStream_t stream) {
  int rh = 2;
  if (a.q.K <= 2048) rh = a.q.rp * a.q.K < (1 << 20) ? 2 : 4;
  else if (a.q.K > 16384 || (a.q.K > 8192 && a.q.rp <= 2 * dev.cus)) rh = 1;
  switch (rh) {
    case 1: return launch_rows_grouped<1>(a, dev, stream);
    case 2: return launch_rows_grouped<2>(a, dev, stream);
    default: return launch_rows_grouped<4>(a, dev, stream);
  }
}

}  // namespace mm
