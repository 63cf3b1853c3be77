// Row kernels of the 8-bit layers: the root-mean-square norm with the
// residual's addition, and the quantiser of activations and weights.
#include "ff_common.cuh"
#include "ff_q8.cuh"

namespace ff {

namespace {

// Sum over a block of 256 threads; every thread gets it.
__device__ __forceinline__ float block_sum(float v, float* red) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < 8; ++w) s += red[w];
  return s;
}

// One block per row, the fp32 row in shared memory.
template <class T>
__global__ void __launch_bounds__(256) k_rms_norm(int C, const __grid_constant__ RmsArgs a) {
  extern __shared__ float row[];
  __shared__ float red[8];
  const long long r = blockIdx.x;
  const T* x = reinterpret_cast<const T*>(a.x) + r * a.ldx;
  const T* rs = reinterpret_cast<const T*>(a.resid) + r * a.ldr;
  T* sm = reinterpret_cast<T*>(a.sum) + r * a.ldsum;
  const T* w = reinterpret_cast<const T*>(a.weight);
  float ss = 0.f;
  for (int c = threadIdx.x; c < C; c += 256) {
    float h = to_f(x[c]);
    if (a.resid) h += to_f(rs[c]);
    if (a.sum) sm[c] = from_f<T>(h);
    row[c] = h;
    ss = fmaf(h, h, ss);
  }
  const float rstd = rsqrtf(block_sum(ss, red) / (float)C + a.eps);
  if (a.out) {
    T* o = reinterpret_cast<T*>(a.out) + r * a.ldo;
    for (int c = threadIdx.x; c < C; c += 256) o[c] = from_f<T>(row[c] * rstd * (w ? to_f(w[c]) : 1.f));
    return;
  }
  // a warp per block of 128 columns
  const int lane = threadIdx.x & 31;
  for (int b = threadIdx.x >> 5; b * 128 < C; b += 8) {
    float v[4];
    uint32_t m = 0;
    for (int i = 0; i < 4; ++i) {
      const int c = b * 128 + 32 * i + lane;
      v[i] = c < C ? row[c] * rstd * (w ? to_f(w[c]) : 1.f) : 0.f;
      m = max(m, abs_bits(v[i]));
    }
    m = __reduce_max_sync(0xffffffffu, m);
    const float s = q8_scale(m), inv = 1.f / s;
    uint8_t* q = reinterpret_cast<uint8_t*>(a.q8.q) + r * a.q8.ldq;
    for (int i = 0; i < 4; ++i) {
      const int c = b * 128 + 32 * i + lane;
      if (c < C) q[c] = (uint8_t)to_e4m3x2(v[i] * inv, 0.f);
    }
    if (lane == 0) a.q8.scale[b * a.q8.lds + r] = s;
  }
}

// TILE rows x 128 columns to a block of 128 threads, a thread per column.
template <class T, int TILE>
__global__ void __launch_bounds__(128) k_quant8(long long rows, int C, const T* x, long long ldx, const Quant8Out o) {
  __shared__ uint32_t red[4];
  const int c = blockIdx.y * 128 + threadIdx.x;
  const long long r0 = (long long)blockIdx.x * TILE;
  const int n = (int)min((long long)TILE, rows - r0);
  uint32_t m = 0;
  if (c < C)
    for (int i = 0; i < n; ++i) m = max(m, abs_bits(to_f(x[(r0 + i) * ldx + c])));
  m = __reduce_max_sync(0xffffffffu, m);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m;
  __syncthreads();
  m = max(max(red[0], red[1]), max(red[2], red[3]));
  const float s = q8_scale(m), inv = 1.f / s;
  if (c < C)
    for (int i = 0; i < n; ++i)
      reinterpret_cast<uint8_t*>(o.q)[(r0 + i) * o.ldq + c] = (uint8_t)to_e4m3x2(to_f(x[(r0 + i) * ldx + c]) * inv, 0.f);
  if (threadIdx.x == 0) o.scale[TILE == 1 ? blockIdx.y * o.lds + r0 : (long long)blockIdx.x * o.lds + blockIdx.y] = s;
}

template <class T>
cudaError_t rms_norm(long long rows, int C, const RmsArgs& a, cudaStream_t s) {
  const size_t smem = (size_t)C * 4;
  const cudaError_t e = cudaFuncSetAttribute(k_rms_norm<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, 32768 * 4);
  if (e != cudaSuccess) return e;
  k_rms_norm<T><<<(unsigned)rows, 256, smem, s>>>(C, a);
  return launched();
}

template <class T>
cudaError_t quant8(int tile, long long rows, int C, const void* x, long long ldx, const Quant8Out& o, cudaStream_t s) {
  const int nb = (C + 127) / 128;
  if (nb > 65535) return cudaErrorInvalidValue;
  if (tile == 1)
    k_quant8<T, 1><<<dim3((unsigned)rows, nb), 128, 0, s>>>(rows, C, (const T*)x, ldx, o);
  else
    k_quant8<T, 128><<<dim3((unsigned)((rows + 127) / 128), nb), 128, 0, s>>>(rows, C, (const T*)x, ldx, o);
  return launched();
}

}  // namespace

cudaError_t launch_rms_norm(DType dt, long long rows, int C, const RmsArgs& a, cudaStream_t s) {
  if (rows <= 0) return cudaSuccess;
  return dt == F32 ? rms_norm<float>(rows, C, a, s) : rms_norm<bf16>(rows, C, a, s);
}

cudaError_t launch_quant8(DType dt, int tile, long long rows, int cols, const void* x, long long ldx,
                          const Quant8Out& o, cudaStream_t s) {
  if (rows <= 0) return cudaSuccess;
  return dt == F32 ? quant8<float>(tile, rows, cols, x, ldx, o, s) : quant8<bf16>(tile, rows, cols, x, ldx, o, s);
}

}  // namespace ff
