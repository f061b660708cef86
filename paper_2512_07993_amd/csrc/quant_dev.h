// Device-side helpers of the 8-bit cache: e4m3 codes (OCP) with a power-of-two scale per block.
#pragma once

#include "scan_dev.h"

namespace skipkv {

// A scale byte e stands for 2^(e - 127): its fp32 bit pattern is e << 23.
__device__ __forceinline__ float scale_of_byte(uint32_t e) { return __uint_as_float(e << 23); }

// Least byte e in 1 .. 254 with amax <= 448 * 2^(e - 127).  448 = 1.75 * 2^8: with amax = f * 2^x, 1 <= f < 2, that is
// x - 8, or x - 7 where f > 1.75.
__device__ __forceinline__ int scale_byte_for(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);  // biased exponent of amax (0 below the normals)
  return min(max(e, 1), 254);
}

// Two fp32 -> two e4m3 codes in the low or high half of `old`, nearest even.  The caller keeps magnitudes at or below 448.
template <bool HIGH>
__device__ __forceinline__ uint32_t to_e4m3(float x, float y, uint32_t old) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, y, (int)old, HIGH);
}
__device__ __forceinline__ float finite_or_nan(float x) {
  return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u ? __uint_as_float(0x7FC00000u) : x;
}

// Two codes of the low or high half of w, scaled, as bf16 (exact: 4 significant bits).
template <bool HIGH>
__device__ __forceinline__ uint32_t e4m3_to_bf16x2(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HIGH));
}

}  // namespace skipkv
