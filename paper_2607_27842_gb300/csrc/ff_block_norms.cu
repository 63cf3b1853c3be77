// The norms at the end of a block and at the beginning of the next one, with gate and
// residual between them (formulas: featfix_op_block_norms).
#include "ff_kv8.cuh"

namespace ff {

namespace {

__device__ __forceinline__ float block_sum(float v, float* red) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.f;
  for (int k = 0; k < 8; ++k) v += red[k];
  return v;
}

// A block to a row, the fp32 row in shared memory.
template <class T>
__global__ void __launch_bounds__(256) k_block_norms(int C, const __grid_constant__ BlockNormsArgs a) {
  extern __shared__ float row[];
  __shared__ float red[8];
  const long long r = blockIdx.x, s = r / a.rpb;
  const T* y = reinterpret_cast<const T*>(a.y) + r * a.ldy;
  const T* x = reinterpret_cast<const T*>(a.x) + r * a.ldx;
  const T *wa = reinterpret_cast<const T*>(a.weight_after), *w = reinterpret_cast<const T*>(a.weight);
  pdl_trigger();
  pdl_wait();
  auto norm = [&] {   // of the row: its mean and 1 / root mean square
    float mean = 0.f, ss = 0.f;
    if (a.centered) {
      for (int c = threadIdx.x; c < C; c += 256) mean += row[c];
      mean = block_sum(mean, red) / C;
    }
    for (int c = threadIdx.x; c < C; c += 256) ss = fmaf(row[c] - mean, row[c] - mean, ss);
    return make_float2(mean, rsqrtf(block_sum(ss, red) / C + a.eps));
  };
  for (int c = threadIdx.x; c < C; c += 256) row[c] = to_f(y[c]);
  if (a.norm_after) {
    const float2 n = norm();
    for (int c = threadIdx.x; c < C; c += 256) row[c] = (row[c] - n.x) * n.y * (wa ? to_f(wa[c]) : 1.f);
  }
  for (int c = threadIdx.x; c < C; c += 256) {
    float h = row[c];
    if (a.gate) h *= a.gate[s * a.gate_stride + c];
    if (a.x) h = fmaf(a.resid_scale, to_f(x[c]), h);
    row[c] = h;
    if (a.sum) reinterpret_cast<T*>(a.sum)[r * a.ldsum + c] = from_f<T>(h);
  }
  if (!a.out && !a.q8.q) return;
  const float2 n = norm();
  for (int c = threadIdx.x; c < C; c += 256) {
    float z = (row[c] - n.x) * n.y * (w ? to_f(w[c]) : 1.f);
    if (a.scale) z *= 1.f + a.scale[s * a.scale_stride + c];
    if (a.shift) z += a.shift[s * a.shift_stride + c];
    row[c] = z;
    if (a.out) reinterpret_cast<T*>(a.out)[r * a.ldo + c] = from_f<T>(z);
  }
  if (a.out) return;
  __syncthreads();
  const int lane = threadIdx.x & 31;
  for (int b = threadIdx.x >> 5; b * 128 < C; b += 8) {
    float m = 0.f;
    for (int c = b * 128 + lane; c < min(C, b * 128 + 128); c += 32) m = max_abs(m, row[c]);
    const float q = q8_scale(__reduce_max_sync(0xffffffffu, __float_as_uint(m))), inv = q8_inv(q);
    for (int c = b * 128 + lane; c < min(C, b * 128 + 128); c += 32)
      reinterpret_cast<uint8_t*>(a.q8.q)[r * a.q8.ldq + c] = (uint8_t)to_e4m3x2(row[c] * inv, 0.f);
    if (lane == 0) a.q8.scale[b * a.q8.lds + r] = q;
  }
}

}  // namespace

cudaError_t launch_block_norms(DType dt, long long rows, int C, const BlockNormsArgs& a, cudaStream_t s) {
  const size_t smem = (size_t)C * 4;
  const void* f = dt == F32 ? (const void*)k_block_norms<float> : (const void*)k_block_norms<bf16>;
  cudaError_t e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, BLOCK_NORMS_COLS_MAX * 4);
  if (e != cudaSuccess) return e;
  e = dt == F32 ? launch_pdl(k_block_norms<float>, (unsigned)rows, 256, smem, s, C, a)
                : launch_pdl(k_block_norms<bf16>, (unsigned)rows, 256, smem, s, C, a);
  return e != cudaSuccess ? e : launched();
}

}  // namespace ff
