// Shared pieces of the quantising kernels (gfx950): one 32-channel block's scale
// and codes, and the LDS gather.
#pragma once

#include "kernels.hpp"

namespace mm {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x32 __attribute__((ext_vector_type(32)));
typedef short i16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef int i32x6 __attribute__((ext_vector_type(6)));
typedef uint32_t u32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

typedef float f32x2 __attribute__((ext_vector_type(2)));

// LDS pointers built from 32-bit byte addresses (the base already added)
typedef const __attribute__((address_space(3))) uint16_t lds_u16_t;

__device__ __forceinline__ uint16_t lds_u16(uint32_t byte_addr) {
  return *reinterpret_cast<lds_u16_t*>((uintptr_t)byte_addr);
}

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t,
                            __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

__device__ __forceinline__ uint32_t min_u16x2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t,
                            __builtin_elementwise_min(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// Zero codes and scale byte for block j of step `step` of row n (padding).
template <int G>
__device__ __forceinline__ void zero_block(const QuantArgs& a, int64_t step, int64_t gstep, int64_t n, int j) {
  uint8_t* dst = a.q[G] + code_offset<G>(step, a.rp, n, j);
  if constexpr (G == 0) {
    *reinterpret_cast<uint4*>(dst) = make_uint4(0u, 0u, 0u, 0u);
  } else if constexpr (G == 1) {
    uint2* d = reinterpret_cast<uint2*>(dst);
    d[0] = d[1] = d[2] = make_uint2(0u, 0u);
  } else {
    *reinterpret_cast<uint4*>(dst) = make_uint4(0u, 0u, 0u, 0u);
    *reinterpret_cast<uint4*>(dst + 512) = make_uint4(0u, 0u, 0u, 0u);
  }
  a.sc[(gstep * a.rp + n) * kStepBlocks + j] = 0;
}

template <int G>
__device__ __forceinline__ void zero_tail(const QuantArgs& a, int64_t step, int64_t gstep, int64_t n, int j) {
  for (int jj = j + 1; jj < kStepBlocks; ++jj) zero_block<G>(a, step, gstep, n, jj);
}

// Bytes from row 0's codes of a block to row n's, n a multiple of the rows per
// pass: whole row groups, then rows within one.
template <int G>
__device__ __forceinline__ int64_t row_offset(int64_t n) {
  return (n & ~(int64_t)(kRowGroup - 1)) * step_row_bytes(G) + (n & (kRowGroup - 1)) * (G == 1 ? 24 : 16);
}

// Quantise the 32 gathered channels d (bf16 pairs) of block b (local to its
// group) of row n = n0 + prow, n0 uniform over the workgroup; dst and sdst are
// the block's codes and scale byte of row prow.  Rows past a.rows are padding
// and quantise an all-zero block.  The thread that owns a group's last block
// also zeroes the padding blocks of that step.
__device__ __forceinline__ void encode_block(uint32_t (&d)[16], int group, bool last, const QuantArgs& a, int64_t n0,
                                             int prow, int b, int gstep0, uint8_t* dst, uint8_t* sdst) {
  const int64_t n = n0 + prow;
  const bool pad_row = n >= a.rows;
#pragma unroll
  for (int i = 0; i < 16; ++i) d[i] = pad_row ? 0u : d[i];

  // absmax: bf16 magnitudes compare as unsigned integers
  uint32_t m[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) m[i] = d[i] & 0x7FFF7FFFu;
#pragma unroll
  for (int i = 4; i < 16; ++i) m[i & 3] = max_u16x2(m[i & 3], d[i] & 0x7FFF7FFFu);
  m[0] = max_u16x2(max_u16x2(m[0], m[1]), max_u16x2(m[2], m[3]));
  const uint32_t amax = (m[0] & 0xFFFFu) > (m[0] >> 16) ? (m[0] & 0xFFFFu) : (m[0] >> 16);

  // Shared exponent e = floor(log2 amax) - emax, clamped below at -127: for
  // a bf16 amax with biased exponent E this is max(E - 127 - emax, -127); a
  // subnormal or zero amax (E = 0) lands on the clamp.  The E8M0 byte is e+127.
  const bool e2m3 = (a.fs & 1) != 0, e5m2 = (a.fs & 2) != 0;  // the alternative formats of groups 1 and 2
  const int emax = group == 0 ? 2 : (group == 1 ? (e2m3 ? 2 : 4) : (e5m2 ? 15 : 8));
  const int E = (int)(amax >> 7);
  const uint32_t sbyte = (uint32_t)(E - emax > 0 ? E - emax : 0);
  // the conversions read the scale's E8M0 exponent from an fp32 operand
  const float scale = __uint_as_float(sbyte << 23);

  const int64_t step = b >> 2;
  const int j = b & 3;
  const int64_t gstep = gstep0 + step;
  sdst[n0 * kStepBlocks] = (uint8_t)sbyte;
  if (group == 0) {
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint32_t v = 0;
      v = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(v, __builtin_bit_cast(bf16x2, d[4 * q + 0]), scale, 0);
      v = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(v, __builtin_bit_cast(bf16x2, d[4 * q + 1]), scale, 1);
      v = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(v, __builtin_bit_cast(bf16x2, d[4 * q + 2]), scale, 2);
      v = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(v, __builtin_bit_cast(bf16x2, d[4 * q + 3]), scale, 3);
      w[q] = v;
    }
    *reinterpret_cast<uint4*>(dst + row_offset<0>(n0)) = make_uint4(w[0], w[1], w[2], w[3]);
    if (last) zero_tail<0>(a, step, gstep, n, j);
  } else if (group == 1) {
    u32x16 v;
    i32x6 c;
    if (e2m3) {
      // clamp the magnitudes to the largest E2M3 value, 7.5 * 2^e (exact in
      // bf16: biased exponent e + 129 = sbyte + 2, mantissa 0x70), keep the
      // signs; nothing then depends on how the conversion treats larger values
      const uint32_t lim = ((sbyte + 2u) << 7) | 0x70u;
      const uint32_t lim2 = lim | (lim << 16);
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = min_u16x2(d[i] & 0x7FFF7FFFu, lim2) | (d[i] & 0x80008000u);
      c = __builtin_amdgcn_cvt_scalef32_pk32_fp6_bf16(__builtin_bit_cast(bf16x32, v), scale);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = d[i];
      c = __builtin_amdgcn_cvt_scalef32_pk32_bf6_bf16(__builtin_bit_cast(bf16x32, v), scale);
    }
    uint2* p = reinterpret_cast<uint2*>(dst + row_offset<1>(n0));
    p[0] = make_uint2((uint32_t)c[0], (uint32_t)c[1]);
    p[1] = make_uint2((uint32_t)c[2], (uint32_t)c[3]);
    p[2] = make_uint2((uint32_t)c[4], (uint32_t)c[5]);
    if (last) zero_tail<1>(a, step, gstep, n, j);
  } else {
    // the largest finite value times 2^e in bf16, mantissa 0x60 (1.75): E4M3
    // 448 (biased exponent e + 127 + 8 = sbyte + 8), E5M2 57344 (sbyte + 15)
    const uint32_t lim = ((sbyte + (e5m2 ? 15u : 8u)) << 7) | 0x60u;
    const uint32_t lim2 = lim | (lim << 16);
    uint32_t w[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      // clamp the magnitudes, keep the signs
      const uint32_t c0 = min_u16x2(d[2 * q] & 0x7FFF7FFFu, lim2) | (d[2 * q] & 0x80008000u);
      const uint32_t c1 = min_u16x2(d[2 * q + 1] & 0x7FFF7FFFu, lim2) | (d[2 * q + 1] & 0x80008000u);
      i16x2 v = {0, 0};
      if (e5m2) {
        v = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(v, __builtin_bit_cast(bf16x2, c0), scale, false);
        v = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(v, __builtin_bit_cast(bf16x2, c1), scale, true);
      } else {
        v = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(v, __builtin_bit_cast(bf16x2, c0), scale, false);
        v = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(v, __builtin_bit_cast(bf16x2, c1), scale, true);
      }
      w[q] = __builtin_bit_cast(uint32_t, v);
    }
    uint8_t* p = dst + row_offset<2>(n0);
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    *reinterpret_cast<uint4*>(p + 512) = make_uint4(w[4], w[5], w[6], w[7]);
    if (last) zero_tail<2>(a, step, gstep, n, j);
  }
}

// base + one 16-bit half of w (one instruction; written out because the
// compiler would otherwise hoist the 32 halves, or their sums, out of the
// loop over the passes and spill).
template <int H>
__device__ __forceinline__ uint32_t add_word(uint32_t base, uint32_t w) {
  uint32_t r;
  if constexpr (H == 0)
    asm("v_add_u32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:WORD_0"
        : "=v"(r)
        : "v"(base), "v"(w));
  else
    asm("v_add_u32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:WORD_1"
        : "=v"(r)
        : "v"(base), "v"(w));
  return r;
}

// 32-bit LDS addresses
template <typename T>
__device__ __forceinline__ T lds_load(uint32_t addr) {
  return *reinterpret_cast<const __attribute__((address_space(3))) T*>((uintptr_t)addr);
}
template <typename T>
__device__ __forceinline__ void lds_store(uint32_t addr, T v) {
  *reinterpret_cast<__attribute__((address_space(3))) T*>((uintptr_t)addr) = v;
}

}  // namespace
}  // namespace mm
