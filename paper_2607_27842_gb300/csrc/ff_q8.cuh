// The 8-bit format of featfix_ops.h: e4m3 values with a scale for each block.
#pragma once

#include <cuda_fp8.h>
#include <stdint.h>

namespace ff {

// Magnitudes compare as their bits do; a NaN is above infinity, so a block's
// maximum carries both on into its scale (fmaxf would drop the NaN).
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Scale of a block from the bits of its largest magnitude.  The least scale,
// 2^-100, keeps 1 / scale finite for blocks of zeros and of denormals.
__device__ __forceinline__ float q8_scale(uint32_t amax_bits) {
  const float s = __uint_as_float(amax_bits) * (1.0f / 448.0f);
  return s < 0x1p-100f ? 0x1p-100f : s;
}

// The larger magnitude, NaN where either is (one instruction, the magnitudes are
// operand modifiers); its bits are ordered as above.
__device__ __forceinline__ float max_abs(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)));
  return r;
}

// 1 / scale within an ulp: it only decides codes that lie within 2^-23 of a tie
// (scales are 2^-100 to 2^120, infinite or NaN, so no result is denormal).
__device__ __forceinline__ float q8_inv(float s) { return __fdividef(1.f, s); }

// Two values in e4m3, rounded to nearest even, past 448 saturated (a rounded
// 1 / scale can lift a block's largest value a half step above 448), a in the low byte.
__device__ __forceinline__ uint32_t to_e4m3x2(float a, float b) {
  return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) {
  return to_e4m3x2(a, b) | to_e4m3x2(c, d) << 16;
}

}  // namespace ff
