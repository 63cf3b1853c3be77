// 8-bit dense layers with a scale for each block of 128.
#include "ff_common.cuh"
#include "ff_q8.cuh"

namespace ff {

namespace {

__device__ __forceinline__ float from_e4m3(uint8_t q) {
  return __half2float(__half(__nv_cvt_fp8_to_halfraw(q, __NV_E4M3)));
}

// 32 rows x 128 columns to a block, 4 x 4 results to a thread.
template <class T>
__global__ void __launch_bounds__(256) k_gemm8(int M, int N, int K, const __grid_constant__ Gemm8Args g) {
  __shared__ float sa[32][33], sw[128][33];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const int m0 = blockIdx.y * 32, n0 = blockIdx.x * 128;
  float acc[4][4] = {};
  for (int b = 0; b * 128 < K; ++b) {
    float part[4][4] = {};
    for (int k0 = b * 128; k0 < min(K, b * 128 + 128); k0 += 32) {
      __syncthreads();
      for (int i = ty; i < 32; i += 8)
        sa[i][tx] = m0 + i < M && k0 + tx < K
                        ? from_e4m3(reinterpret_cast<const uint8_t*>(g.a)[(m0 + i) * g.lda + k0 + tx]) : 0.f;
      for (int i = ty; i < 128; i += 8)
        sw[i][tx] = n0 + i < N && k0 + tx < K
                        ? from_e4m3(reinterpret_cast<const uint8_t*>(g.w)[(n0 + i) * g.ldw + k0 + tx]) : 0.f;
      __syncthreads();
      for (int k = 0; k < 32; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) part[i][j] = fmaf(sa[ty * 4 + i][k], sw[tx + 32 * j][k], part[i][j]);
    }
    const float fw = g.sw[blockIdx.x * g.ldsw + b];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int m = m0 + ty * 4 + i;
      const float f = m < M ? g.sa[b * g.ldsa + m] * fw : 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(f, part[i][j], acc[i][j]);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const long long m = m0 + ty * 4 + i;
    if (m >= M) return;
    uint32_t mx = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + tx + 32 * j;
      float y = acc[i][j];
      if (n < N) {
        if (g.bias) y += to_f(reinterpret_cast<const T*>(g.bias)[n]);
        if (g.act) y = gelu_tanh(y);
        if (g.gate) y *= g.gate[m / g.rpb * g.gate_stride + n];
        if (g.resid) y += to_f(reinterpret_cast<const T*>(g.resid)[m * g.ldr + n]);
        if (g.out) reinterpret_cast<T*>(g.out)[m * g.ldo + n] = from_f<T>(y);
        mx = max(mx, abs_bits(y));
      }
      acc[i][j] = y;
    }
    if (!g.out) {
      const float s = q8_scale(__reduce_max_sync(0xffffffffu, mx)), inv = 1.f / s;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (n0 + tx + 32 * j < N)
          reinterpret_cast<uint8_t*>(g.q8.q)[m * g.q8.ldq + n0 + tx + 32 * j] = (uint8_t)to_e4m3x2(acc[i][j] * inv, 0.f);
      if (tx == 0) g.q8.scale[blockIdx.x * g.q8.lds + m] = s;
    }
  }
}

}  // namespace

cudaError_t gemm8(DType dt, int M, int N, int K, const Gemm8Args& g, cudaStream_t s) {
  if (M <= 0) return cudaSuccess;
  const dim3 grid((N + 127) / 128, (M + 31) / 32);
  if (grid.y > 65535) return cudaErrorInvalidValue;
  if (dt == F32)
    k_gemm8<float><<<grid, 256, 0, s>>>(M, N, K, g);
  else
    k_gemm8<bf16><<<grid, 256, 0, s>>>(M, N, K, g);
  return launched();
}

}  // namespace ff
