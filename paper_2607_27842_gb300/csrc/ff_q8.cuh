// Declarations shared by the kernels of the 8-bit layers and their C entries, and the
// 8-bit format of featfix_ops.h: e4m3 values with a scale for each block.
#pragma once

#include "ff_common.cuh"

#include <cuda_fp8.h>
#include <stdint.h>

namespace ff {

// 8-bit layers (formats and formulas: featfix_ops.h)
struct Quant8Out {   // an 8-bit tensor and its scales
  void* q;
  long long ldq;
  float* scale;
  long long lds;
};
constexpr int RMS_COLS_MAX = 32768;   // widest row of the norm
struct RmsArgs {
  const void* x; long long ldx;
  const void* resid; long long ldr;   // nullable
  void* sum; long long ldsum;         // nullable
  const void* weight;                 // nullable
  float eps;
  void* out; long long ldo;           // null: q8
  Quant8Out q8;
};
cudaError_t launch_rms_norm(DType dt, long long rows, int C, const RmsArgs& a, cudaStream_t s);
cudaError_t launch_quant8(DType dt, int tile, long long rows, int cols, const void* x, long long ldx,
                          const Quant8Out& o, cudaStream_t s);
constexpr int ROPE_PAIRS = 128;   // head widths up to 256
struct RopeSide {
  const void* x; long long ldx;
  void* out; long long ldo;
  const void* weight;   // nullable: no norm
  int heads;
};
struct RopeArgs {
  RopeSide side[2];     // q, k
  const int* pos;
  long long ld_pos;
  int hd, rot, halves;
  float eps;
  // turns per position of every pair (negative: the inverse), as an unevaluated
  // sum of two floats, and the pair's axis
  float2 freq[ROPE_PAIRS];
  unsigned char axis[ROPE_PAIRS];
};
cudaError_t launch_rope(DType dt, long long rows, const RopeArgs& a, cudaStream_t s);
struct Gemm8Args {
  const void* a; long long lda;
  const float* sa; long long ldsa;
  const void* w; long long ldw;
  const float* sw; long long ldsw;
  const void* bias;                    // nullable, [N]
  int act;
  const float* gate; long long gate_stride; int rpb;   // nullable
  const void* resid; long long ldr;    // nullable
  void* out; long long ldo;            // null: q8
  Quant8Out q8;
};
cudaError_t gemm8(DType dt, int M, int N, int K, const Gemm8Args& g, cudaStream_t s);
// The watchdog flags of gemm8's kernels, cleared; waits for the device.
cudaError_t gemm8_watchdog_take(unsigned int* flags);
// Lets a part of both bounded waits run out; their limits, from what it took.
cudaError_t gemm8_watchdog_probe(unsigned long long (&limit_ns)[2]);

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
