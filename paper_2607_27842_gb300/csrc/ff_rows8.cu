// Row kernels of the 8-bit layers: the root-mean-square norm with the residual's
// addition (formula: featfix_op_rms_norm), and the quantiser of activations and
// weights.  Both are bound by memory: every element is read once into registers, and
// what is written is computed from there.
#include "ff_common.cuh"
#include "ff_q8.cuh"

#include <algorithm>

namespace ff {

namespace {

// Four elements of a lane's share of a 128-column block: adjacent columns 4 lane ..
// in one vector where rows allow it, columns lane, lane + 32, .. otherwise.
template <class T, bool VEC> struct Four;
template <> struct Four<float, true> {
  float4 r;
  __device__ __forceinline__ void load(const float* p, int lane, int) { r = *reinterpret_cast<const float4*>(p + 4 * lane); }
  __device__ __forceinline__ void get(float (&v)[4]) const { v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w; }
  static __device__ __forceinline__ void store(float* p, int lane, int, const float (&v)[4]) {
    *reinterpret_cast<float4*>(p + 4 * lane) = make_float4(v[0], v[1], v[2], v[3]);
  }
};
template <> struct Four<bf16, true> {
  uint2 r;
  __device__ __forceinline__ void load(const bf16* p, int lane, int) { r = *reinterpret_cast<const uint2*>(p + 4 * lane); }
  __device__ __forceinline__ void get(float (&v)[4]) const {
    const f32x2 a = bf2u(r.x), b = bf2u(r.y);
    v[0] = lo_f(a); v[1] = hi_f(a); v[2] = lo_f(b); v[3] = hi_f(b);
  }
  static __device__ __forceinline__ void store(bf16* p, int lane, int, const float (&v)[4]) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
    *reinterpret_cast<uint2*>(p + 4 * lane) =
        make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
  }
};
template <class T> struct Four<T, false> {
  T r[4];
  __device__ __forceinline__ void load(const T* p, int lane, int n) {
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = lane + 32 * k < n ? p[lane + 32 * k] : from_f<T>(0.f);
  }
  __device__ __forceinline__ void get(float (&v)[4]) const {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = to_f(r[k]);
  }
  static __device__ __forceinline__ void store(T* p, int lane, int n, const float (&v)[4]) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (lane + 32 * k < n) p[lane + 32 * k] = from_f<T>(v[k]);
  }
};
// the four as e4m3 (p: the block's first byte, 16-byte aligned rows of bytes)
template <bool VEC>
__device__ __forceinline__ void store8(uint8_t* p, int lane, int n, const float (&v)[4], float inv) {
  const uint32_t c = to_e4m3x4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
  if (VEC) {
    *reinterpret_cast<uint32_t*>(p + 4 * lane) = c;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (lane + 32 * k < n) p[lane + 32 * k] = (uint8_t)(c >> (8 * k));
  }
}
__device__ __forceinline__ uint32_t amax4(const float (&v)[4]) {
  return __reduce_max_sync(0xffffffffu, max(max(abs_bits(v[0]), abs_bits(v[1])), max(abs_bits(v[2]), abs_bits(v[3]))));
}

// W warps to a row (1, 2, 4 or 8; eight warps to a block), NB 128-column blocks to a
// warp: block i of warp w is w + W i.  A lane has four columns of each, so one warp
// instruction finds a block's largest magnitude.  With VEC, C is a multiple of 4: a
// lane's four columns are all in the row or none is.
template <class T, int NB, bool VEC, bool NORM, bool Q8>
__global__ void __launch_bounds__(256) k_rows8(long long rows, int C, int W, const __grid_constant__ RmsArgs a) {
  __shared__ float red[8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int w = warp & (W - 1);
  const long long r = (long long)blockIdx.x * (8 / W) + warp / W;
  const bool on = r < rows;
  const T* x = reinterpret_cast<const T*>(a.x) + r * a.ldx;
  Four<T, VEC> f[NB], g[NB];
  pdl_trigger();
  pdl_wait();
  auto in = [&](int i) { return on && (w + W * i) * 128 + (VEC ? 4 * lane : lane) < C; };
#pragma unroll
  for (int i = 0; i < NB; ++i)
    if (in(i)) f[i].load(x + (w + W * i) * 128, lane, C - (w + W * i) * 128);
  if (NORM && a.resid) {
    const T* rs = reinterpret_cast<const T*>(a.resid) + r * a.ldr;
#pragma unroll
    for (int i = 0; i < NB; ++i)
      if (in(i)) g[i].load(rs + (w + W * i) * 128, lane, C - (w + W * i) * 128);
  }
  float h[NB][4], ss = 0.f;
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    if (in(i)) {
      f[i].get(h[i]);
      if (NORM && a.resid) {
        float u[4];
        g[i].get(u);
#pragma unroll
        for (int k = 0; k < 4; ++k) h[i][k] += u[k];
      }
      if (NORM) {
#pragma unroll
        for (int k = 0; k < 4; ++k) ss = fmaf(h[i][k], h[i][k], ss);
        if (a.sum)
          Four<T, VEC>::store(reinterpret_cast<T*>(a.sum) + r * a.ldsum + (w + W * i) * 128, lane, C - (w + W * i) * 128, h[i]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) h[i][k] = 0.f;
    }
  }
  float rstd = 1.f;
  if (NORM) {
    const T* wt = reinterpret_cast<const T*>(a.weight);
    if (wt) {   // (its loads are under way during the sum)
#pragma unroll
      for (int i = 0; i < NB; ++i)
        if (in(i)) f[i].load(wt + (w + W * i) * 128, lane, C - (w + W * i) * 128);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (W > 1) {
      if (lane == 0) red[warp] = ss;
      __syncthreads();
      ss = 0.f;
      for (int k = 0; k < W; ++k) ss += red[warp - w + k];
    }
    rstd = rsqrtf(ss / (float)C + a.eps);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      float u[4] = {1.f, 1.f, 1.f, 1.f};
      if (wt && in(i)) f[i].get(u);
#pragma unroll
      for (int k = 0; k < 4; ++k) h[i][k] = h[i][k] * rstd * u[k];
    }
  }
  if constexpr (!Q8) {
#pragma unroll
    for (int i = 0; i < NB; ++i)
      if (in(i))
        Four<T, VEC>::store(reinterpret_cast<T*>(a.out) + r * a.ldo + (w + W * i) * 128, lane, C - (w + W * i) * 128, h[i]);
  } else {
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int b = w + W * i;
      if (!on || b * 128 >= C) continue;   // (warp-uniform)
      // columns past the row's end hold no magnitude, not even a NaN's
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (b * 128 + (VEC ? 4 * lane : lane + 32 * k) >= C) h[i][k] = 0.f;
      const float s = q8_scale(amax4(h[i]));
      if (in(i)) store8<VEC>(reinterpret_cast<uint8_t*>(a.q8.q) + r * a.q8.ldq + b * 128, lane, C - b * 128, h[i], 1.f / s);
      if (lane == 0) a.q8.scale[b * a.q8.lds + r] = s;
    }
  }
}

// Norm of rows too wide for registers: one block to a row, the fp32 row in shared
// memory.
template <class T>
__global__ void __launch_bounds__(1024) k_rows8_wide(int C, const __grid_constant__ RmsArgs a) {
  extern __shared__ float row[];
  __shared__ float red[32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long r = blockIdx.x;
  const T* x = reinterpret_cast<const T*>(a.x) + r * a.ldx;
  const T* rs = reinterpret_cast<const T*>(a.resid) + r * a.ldr;
  T* sm = reinterpret_cast<T*>(a.sum) + r * a.ldsum;
  const T* w = reinterpret_cast<const T*>(a.weight);
  pdl_trigger();
  pdl_wait();
  float ss = 0.f;
#pragma unroll 4
  for (int c = threadIdx.x; c < C; c += 1024) {
    float h = to_f(x[c]);
    if (a.resid) h += to_f(rs[c]);
    if (a.sum) sm[c] = from_f<T>(h);
    row[c] = h;
    ss = fmaf(h, h, ss);
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
  if (lane == 0) red[warp] = ss;
  __syncthreads();
  ss = 0.f;
  for (int k = 0; k < 32; ++k) ss += red[k];
  const float rstd = rsqrtf(ss / (float)C + a.eps);
  auto y = [&](int c) { return row[c] * rstd * (w ? to_f(w[c]) : 1.f); };
  if (a.out) {
    T* o = reinterpret_cast<T*>(a.out) + r * a.ldo;
    for (int c = threadIdx.x; c < C; c += 1024) o[c] = from_f<T>(y(c));
    return;
  }
  for (int b = warp; b * 128 < C; b += 32) {
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = b * 128 + 32 * k + lane < C ? y(b * 128 + 32 * k + lane) : 0.f;
    const float s = q8_scale(amax4(v));
    store8<false>(reinterpret_cast<uint8_t*>(a.q8.q) + r * a.q8.ldq + b * 128, lane, C - b * 128, v, 1.f / s);
    if (lane == 0) a.q8.scale[b * a.q8.lds + r] = s;
  }
}

// 128 x 128 blocks of a weight: 16 rows to a warp, four columns to a lane.
template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_quant8_tile(long long rows, int C, const T* x, long long ldx, const Quant8Out o) {
  __shared__ uint32_t red[8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int c0 = blockIdx.x * 128, n = C - c0;
  const long long r0 = (long long)blockIdx.y * 128 + warp * 16;
  const bool in = (VEC ? 4 * lane : lane) < n;
  Four<T, VEC> f[16];
  pdl_trigger();
  pdl_wait();
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (in && r0 + i < rows) f[i].load(x + (r0 + i) * ldx + c0, lane, n);
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (in && r0 + i < rows) f[i].get(v);
#pragma unroll
    for (int k = 0; k < 4; ++k) m = max(m, abs_bits(v[k]));
  }
  m = __reduce_max_sync(0xffffffffu, m);
  if (lane == 0) red[warp] = m;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 8; ++k) m = max(m, red[k]);
  const float s = q8_scale(m), inv = 1.f / s;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if (!in || r0 + i >= rows) continue;
    float v[4];
    f[i].get(v);
    store8<VEC>(reinterpret_cast<uint8_t*>(o.q) + (r0 + i) * o.ldq + c0, lane, n, v, inv);
  }
  if (threadIdx.x == 0) o.scale[blockIdx.y * o.lds + blockIdx.x] = s;
}

constexpr int NB_MAX = 16;   // 64 fp32 values to a thread

template <class T, bool VEC, bool NORM, bool Q8>
cudaError_t rows8_nb(int nb, int W, long long rows, int C, const RmsArgs& a, cudaStream_t s) {
  const long long grid = (rows + 8 / W - 1) / (8 / W);
  cudaError_t e;
  if (nb <= 1) e = launch_pdl(k_rows8<T, 1, VEC, NORM, Q8>, (unsigned)grid, 256, 0, s, rows, C, W, a);
  else if (nb <= 2) e = launch_pdl(k_rows8<T, 2, VEC, NORM, Q8>, (unsigned)grid, 256, 0, s, rows, C, W, a);
  else if (nb <= 4) e = launch_pdl(k_rows8<T, 4, VEC, NORM, Q8>, (unsigned)grid, 256, 0, s, rows, C, W, a);
  else if (nb <= 8) e = launch_pdl(k_rows8<T, 8, VEC, NORM, Q8>, (unsigned)grid, 256, 0, s, rows, C, W, a);
  else e = launch_pdl(k_rows8<T, NB_MAX, VEC, NORM, Q8>, (unsigned)grid, 256, 0, s, rows, C, W, a);
  return e != cudaSuccess ? e : launched();
}

// Whether a row pointer and stride keep vectors of four elements aligned.
template <class T> bool al4(const void* p, long long ld) {
  return !((uintptr_t)p & (4 * sizeof(T) - 1)) && ld % 4 == 0;
}

template <class T, bool NORM>
cudaError_t rows8(long long rows, int C, const RmsArgs& a, cudaStream_t s) {
  const int blocks = (C + 127) / 128;
  // Warps to a row: as few as hold it with 16 blocks each, more while the rows alone
  // leave the SMs without 8 warps each (1 x 2048: one block to a warp and the
  // other half of them idle, instead of 16 in one).
  int W = 1;
  while (W < 8 && (blocks > NB_MAX * W || (rows * W < 152 * 8 && blocks > W))) W *= 2;
  const int nb = (blocks + W - 1) / W;
  if constexpr (NORM) {
    if (nb > NB_MAX) {
      const size_t smem = (size_t)C * 4;
      const cudaError_t e = cudaFuncSetAttribute(k_rows8_wide<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
      if (e != cudaSuccess) return e;
      const cudaError_t l = launch_pdl(k_rows8_wide<T>, (unsigned)rows, 1024, smem, s, C, a);
      return l != cudaSuccess ? l : launched();
    }
  }
  const bool vec = C % 4 == 0 && al4<T>(a.x, a.ldx) && (!a.resid || al4<T>(a.resid, a.ldr)) &&
                   (!a.sum || al4<T>(a.sum, a.ldsum)) && (!a.weight || al4<T>(a.weight, 0)) &&
                   (!a.out || al4<T>(a.out, a.ldo));
  if constexpr (NORM) {
    if (a.out)
      return vec ? rows8_nb<T, true, true, false>(nb, W, rows, C, a, s) : rows8_nb<T, false, true, false>(nb, W, rows, C, a, s);
  }
  return vec ? rows8_nb<T, true, NORM, true>(nb, W, rows, C, a, s) : rows8_nb<T, false, NORM, true>(nb, W, rows, C, a, s);
}

template <class T>
cudaError_t quant8(int tile, long long rows, int C, const void* x, long long ldx, const Quant8Out& o, cudaStream_t s) {
  if (tile == 1 && (C + 127) / 128 <= 8 * NB_MAX) {
    RmsArgs a = {};
    a.x = x;
    a.ldx = ldx;
    a.q8 = o;
    return rows8<T, false>(rows, C, a, s);
  }
  if (tile == 1) {   // wider rows than registers hold: runs of columns, each a matrix of its own
    for (int c = 0; c < C; c += 128 * 8 * NB_MAX) {
      const Quant8Out part = {reinterpret_cast<uint8_t*>(o.q) + c, o.ldq, o.scale + (c / 128) * o.lds, o.lds};
      const cudaError_t e = quant8<T>(1, rows, std::min(C - c, 128 * 8 * NB_MAX), reinterpret_cast<const T*>(x) + c, ldx, part, s);
      if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
  }
  // (row blocks in the grid's second dimension, at most 65535 to a launch)
  for (long long r = 0; r < rows; r += 65535 * 128ll) {
    const long long n = std::min(rows - r, 65535 * 128ll);
    const T* xr = reinterpret_cast<const T*>(x) + r * ldx;
    const Quant8Out part = {reinterpret_cast<uint8_t*>(o.q) + r * o.ldq, o.ldq, o.scale + (r / 128) * o.lds, o.lds};
    const dim3 grid((C + 127) / 128, (unsigned)((n + 127) / 128));
    const cudaError_t e = C % 4 == 0 && al4<T>(x, ldx) ? launch_pdl(k_quant8_tile<T, true>, grid, 256, 0, s, n, C, xr, ldx, part)
                                                       : launch_pdl(k_quant8_tile<T, false>, grid, 256, 0, s, n, C, xr, ldx, part);
    if (e != cudaSuccess) return e;
    const cudaError_t l = launched();
    if (l != cudaSuccess) return l;
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_rms_norm(DType dt, long long rows, int C, const RmsArgs& a, cudaStream_t s) {
  if (rows <= 0) return cudaSuccess;
  return dt == F32 ? rows8<float, true>(rows, C, a, s) : rows8<bf16, true>(rows, C, a, s);
}

cudaError_t launch_quant8(DType dt, int tile, long long rows, int cols, const void* x, long long ldx,
                          const Quant8Out& o, cudaStream_t s) {
  if (rows <= 0) return cudaSuccess;
  return dt == F32 ? quant8<float>(tile, rows, cols, x, ldx, o, s) : quant8<bf16>(tile, rows, cols, x, ldx, o, s);
}

}  // namespace ff
