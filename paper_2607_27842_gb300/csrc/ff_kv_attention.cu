// Attention of one new token of each sequence over the 8-bit key-value cache
// (formulas: featfix_op_kv_attention).
#include "ff_kv8.cuh"

#include <cuda_fp16.h>

namespace ff {

namespace {

__device__ __forceinline__ void from_e4m3x8(uint2 u, float (&v)[8]) {
  const uint32_t w[2] = {u.x, u.y};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i / 2] >> (16 * (i & 1))), __NV_E4M3);
    const float2 f = __half22float2(h);
    v[2 * i] = f.x, v[2 * i + 1] = f.y;
  }
}

// A block to a query head of one sequence, a warp to every eighth token, eight columns
// to a lane; running maximum and sum per warp, joined at the end.
template <class T>
__global__ void __launch_bounds__(256) k_kv_attention(const __grid_constant__ KvCache c, const __grid_constant__ KvAttnArgs a) {
  __shared__ float sm[8], sl[8], so[8][KV_DIM_MAX];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, col = 8 * lane;
  const int b = blockIdx.x, j = blockIdx.y, head = j / (a.q_heads / c.heads);
  pdl_trigger();
  pdl_wait();
  const int len = kv_len(c, b), first = a.window && len > a.window ? len - a.window : 0;
  float q[8] = {0, 0, 0, 0, 0, 0, 0, 0}, o[8] = {0, 0, 0, 0, 0, 0, 0, 0}, m = -INFINITY, l = 0.f;
  const bool in = col < c.head_dim;
  if (in) {
    const T* p = reinterpret_cast<const T*>(a.q) + b * a.ldq + (long long)j * c.head_dim + col;
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = to_f(p[i]) * a.scale;
  }
  for (int t = first + warp; t < len; t += 8) {
    const int page = kv_page(c, b, t), slot = t % c.page_size;
    if (page < 0) continue;
    float k[8] = {0, 0, 0, 0, 0, 0, 0, 0}, v[8] = {0, 0, 0, 0, 0, 0, 0, 0}, x = 0.f;
    if (in) {
      from_e4m3x8(*reinterpret_cast<const uint2*>((const uint8_t*)c.k + page * c.k_stride[0] + slot * c.k_stride[1] +
                                                  head * c.k_stride[2] + col), k);
      from_e4m3x8(*reinterpret_cast<const uint2*>((const uint8_t*)c.v + page * c.v_stride[0] + slot * c.v_stride[1] +
                                                  head * c.v_stride[2] + col), v);
    }
    const float ks = kv_scale(c.k_scale[page * c.k_scale_stride[0] + slot * c.k_scale_stride[1] + head * c.k_scale_stride[2]]);
    const float vs = kv_scale(c.v_scale[page * c.v_scale_stride[0] + slot * c.v_scale_stride[1] + head * c.v_scale_stride[2]]);
#pragma unroll
    for (int i = 0; i < 8; ++i) x = fmaf(q[i], k[i], x);
#pragma unroll
    for (int s = 16; s; s >>= 1) x += __shfl_xor_sync(0xffffffffu, x, s);
    x *= ks;
    const float mn = fmaxf(m, x), f = m == -INFINITY ? 0.f : expf(m - mn), p = expf(x - mn), w = p * vs;
    l = l * f + p;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = fmaf(w, v[i], o[i] * f);
    m = mn;
  }
  if (lane == 0) sm[warp] = m, sl[warp] = l;
  if (in)
#pragma unroll
    for (int i = 0; i < 8; ++i) so[warp][col + i] = o[i];
  __syncthreads();
  float top = -INFINITY, sum = 0.f;
  for (int w = 0; w < 8; ++w) top = fmaxf(top, sm[w]);
  for (int w = 0; w < 8; ++w) sum += sm[w] == -INFINITY ? sl[w] : sl[w] * expf(sm[w] - top);
  if (threadIdx.x < c.head_dim) {
    float y = 0.f;
    for (int w = 0; w < 8; ++w) y += sm[w] == -INFINITY ? so[w][threadIdx.x] : so[w][threadIdx.x] * expf(sm[w] - top);
    reinterpret_cast<T*>(a.out)[b * a.ldo + (long long)j * c.head_dim + threadIdx.x] = from_f<T>(sum == 0.f ? 0.f : y / sum);
  }
  if (a.lse && threadIdx.x == 0) a.lse[(long long)b * a.q_heads + j] = top + logf(sum);
}

}  // namespace

size_t kv_attention_workspace(int, int, int, int, long long) { return 0; }

cudaError_t launch_kv_attention(DType dt, const KvCache& c, const KvAttnArgs& a, cudaStream_t s) {
  const dim3 grid(c.seqs, a.q_heads);
  const cudaError_t e = dt == F32 ? launch_pdl(k_kv_attention<float>, grid, 256, 0, s, c, a)
                                  : launch_pdl(k_kv_attention<bf16>, grid, 256, 0, s, c, a);
  return e != cudaSuccess ? e : launched();
}

}  // namespace ff
