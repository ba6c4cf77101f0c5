// Blocks of fp32 or bf16 values to 4-bit codes and scales.
#pragma once
#include "sfc_row_io.h"

namespace sfc {

typedef __bf16 qbf16x2 __attribute__((ext_vector_type(2)));
typedef float qf32x2 __attribute__((ext_vector_type(2)));

// Scale code of a block whose largest magnitude has the fp32 bits `top` (sign bit clear).
__device__ __forceinline__ uint32_t scale_code(uint32_t top) {
  const int field = (int)(top >> 23);
  return field == 255 ? 255u : (uint32_t)(field > 2 ? field - 2 : 0);
}
// The scale as fp32.  255: any finite number (the block is NaN whatever its codes).
__device__ __forceinline__ float scale_value(uint32_t s) {
  return __builtin_bit_cast(float, s == 255 ? 127u << 23 : s == 0 ? 1u << 22 : s << 23);
}

// Largest magnitude (as fp32 bits) of eight elements: magnitudes order as their bits do,
// NaN above all.
template <bool BF16>
__device__ __forceinline__ uint32_t top8(const Raw8<BF16>& r) {
  uint32_t m = 0;
  if constexpr (BF16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = (r.w[0][i] << 16) & 0x7FFFFFFFu, hi = r.w[0][i] & 0x7FFF0000u;
      m = m > lo ? m : lo;
      m = m > hi ? m : hi;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t v = r.w[i >> 2][i & 3] & 0x7FFFFFFFu;
      m = m > v ? m : v;
    }
  }
  return m;
}

// Codes of eight elements, the first in the low bits.
template <bool BF16>
__device__ __forceinline__ uint32_t codes8(const Raw8<BF16>& r, float scale) {
  uint32_t q = 0;
  if constexpr (BF16) {
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(qbf16x2, (uint32_t)r.w[0][0]), scale, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(qbf16x2, (uint32_t)r.w[0][1]), scale, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(qbf16x2, (uint32_t)r.w[0][2]), scale, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(qbf16x2, (uint32_t)r.w[0][3]), scale, 3);
  } else {
    float f[8];
    to_float<BF16>(r, f);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[0], f[1], scale, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[2], f[3], scale, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[4], f[5], scale, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[6], f[7], scale, 3);
  }
  return q;
}

}  // namespace sfc
