// Row kernels of the 8-bit layers: the root-mean-square norm with the residual's
// addition (formula: featfix_op_rms_norm), and the quantiser of activations and
// weights.  Both are bound by memory: every element is read once into registers, and
// what is written is computed from there.
#include "ff_common.cuh"
#include "ff_host.h"
#include "ff_q8.cuh"
#include "ff_rows8.cuh"

#include <algorithm>

namespace ff {

namespace {

// W warps to a row (1, 2, 4 or 8; eight warps to a block), NB adjacent 128-column
// blocks to a warp.  A lane has four columns of each, so one warp instruction finds a
// block's largest magnitude.  With VEC, C is a multiple of 4: a lane's four columns
// are all in the row or none is.  Bound by instruction issue before it was by memory:
// hence the adjacent blocks (one address, constant offsets), packed pairs and
// approximate reciprocals (14566 x 2048 with residual and 8-bit output 45 us without
// them).  Measured there: 34.8 us (6.0 TB/s), bf16 output 35.5 (6.7), the quantiser alone
// 16.6 (5.4, part of it from L2); rows of 1001 (single elements) 26.0 us (3.9).
template <class T, int NB, bool VEC, bool NORM, bool Q8>
__global__ void __launch_bounds__(256) k_rows8(long long rows, int C, int W, const __grid_constant__ RmsArgs a) {
  __shared__ float red[8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int w = warp & (W - 1);
  const long long r = (long long)blockIdx.x * (8 / W) + warp / W;
  const int c0 = w * NB * 128 + at<VEC>(lane), left = r < rows ? C - c0 : 0;   // columns from the lane's first on
  Four<T, VEC> f[NB], g[NB];
  pdl_trigger();
  pdl_wait();
  const T* x = reinterpret_cast<const T*>(a.x) + r * a.ldx + c0;
#pragma unroll
  for (int i = 0; i < NB; ++i)
    if (128 * i < left) f[i].load(x + 128 * i, left - 128 * i);
  if (NORM && a.resid) {
    const T* rs = reinterpret_cast<const T*>(a.resid) + r * a.ldr + c0;
#pragma unroll
    for (int i = 0; i < NB; ++i)
      if (128 * i < left) g[i].load(rs + 128 * i, left - 128 * i);
  }
  f32x2 h[NB][2], s2 = 0;
  T* sm = reinterpret_cast<T*>(a.sum) + r * a.ldsum + c0;
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    h[i][0] = h[i][1] = 0;
    if (128 * i < left) {
      f[i].get(h[i]);
      if (NORM && a.resid) {
        f32x2 u[2];
        g[i].get(u);
        h[i][0] = fadd2(h[i][0], u[0]);
        h[i][1] = fadd2(h[i][1], u[1]);
      }
      if (NORM && a.sum) Four<T, VEC>::store(sm + 128 * i, left - 128 * i, h[i]);
    }
    if (NORM) s2 = ffma2(h[i][1], h[i][1], ffma2(h[i][0], h[i][0], s2));
  }
  if constexpr (NORM) {
    const T* wt = reinterpret_cast<const T*>(a.weight) + c0;
    if (a.weight) {   // (its loads are under way during the sum)
#pragma unroll
      for (int i = 0; i < NB; ++i)
        if (128 * i < left) f[i].load(wt + 128 * i, left - 128 * i);
    }
    float ss = lo_f(s2) + hi_f(s2);
#pragma unroll
    for (int o = 16; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (W > 1) {
      if (lane == 0) red[warp] = ss;
      __syncthreads();
      ss = 0.f;
      for (int k = 0; k < W; ++k) ss += red[warp - w + k];
    }
    const float rstd = rsqrtf(ss / (float)C + a.eps);
    const f32x2 r2 = f2u(rstd, rstd);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      h[i][0] = fmul2(h[i][0], r2);
      h[i][1] = fmul2(h[i][1], r2);
      if (a.weight && 128 * i < left) {
        f32x2 u[2];
        f[i].get(u);
        h[i][0] = fmul2(h[i][0], u[0]);
        h[i][1] = fmul2(h[i][1], u[1]);
      }
    }
  }
  if constexpr (!Q8) {
    T* o = reinterpret_cast<T*>(a.out) + r * a.ldo + c0;
#pragma unroll
    for (int i = 0; i < NB; ++i)
      if (128 * i < left) Four<T, VEC>::store(o + 128 * i, left - 128 * i, h[i]);
  } else {
    uint8_t* q = reinterpret_cast<uint8_t*>(a.q8.q) + r * a.q8.ldq + c0;
    float* sp = a.q8.scale + (long long)(w * NB) * a.q8.lds + r;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      // columns past the row's end hold no magnitude, not even a NaN's
      float m = VEC ? amax4(h[i]) : 0.f;
      if (VEC) {
        if (128 * i >= left) m = 0.f;
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (128 * i + 32 * k < left) m = max_abs(m, k & 1 ? hi_f(h[i][k / 2]) : lo_f(h[i][k / 2]));
      }
      const float s = q8_scale(__reduce_max_sync(0xffffffffu, __float_as_uint(m)));
      if (128 * i < left) store8<VEC>(q + 128 * i, left - 128 * i, h[i], q8_inv(s));
      if (lane == 0 && 128 * i < left) sp[i * a.q8.lds] = s;
    }
  }
}

// Norm of rows too wide for registers: one block to a row, the fp32 row in shared
// memory, element by element (2048 x 20480 bf16 with residual and 8-bit output 123 us, 2.4
// TB/s; the kernel above takes 43 for 16384 columns).
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
    const f32x2 v2[2] = {f2u(v[0], v[1]), f2u(v[2], v[3])};
    const float s = q8_scale(__reduce_max_sync(0xffffffffu, __float_as_uint(amax4(v2))));
    store8<false>(reinterpret_cast<uint8_t*>(a.q8.q) + r * a.q8.ldq + b * 128 + lane, C - b * 128 - lane, v2, q8_inv(s));
    if (lane == 0) a.q8.scale[b * a.q8.lds + r] = s;
  }
}

// 128 x 128 blocks of a weight: 16 rows to a warp, four columns to a lane, all of them
// loaded before the block's maximum is known.  Bound by memory: 8192 x 2048 fp32 13.9 us
// (6.1 TB/s).
template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_quant8_tile(long long rows, int C, const T* x, long long ldx, const Quant8Out o) {
  __shared__ float red[8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int c0 = blockIdx.x * 128 + at<VEC>(lane), left = C - c0;
  const long long r0 = (long long)blockIdx.y * 128 + warp * 16;
  const int n = left > 0 ? (int)max(0ll, min(16ll, rows - r0)) : 0;
  Four<T, VEC> f[16];
  pdl_trigger();
  pdl_wait();
  const T* p = x + r0 * ldx + c0;
#pragma unroll
  for (int i = 0; i < 16; ++i, p += ldx)
    if (i < n) f[i].load(p, left);
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    f32x2 v[2] = {0, 0};
    if (i < n) f[i].get(v);
    m = max_abs(m, amax4(v));
  }
  m = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(m)));
  if (lane == 0) red[warp] = m;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 8; ++k) m = max_abs(m, red[k]);
  const float s = q8_scale(__float_as_uint(m)), inv = q8_inv(s);
  uint8_t* q = reinterpret_cast<uint8_t*>(o.q) + r0 * o.ldq + c0;
#pragma unroll
  for (int i = 0; i < 16; ++i, q += o.ldq) {
    if (i >= n) continue;
    f32x2 v[2];
    f[i].get(v);
    store8<VEC>(q, left, v, inv);
  }
  if (threadIdx.x == 0) o.scale[blockIdx.y * o.lds + blockIdx.x] = s;
}

// blocks to a warp: at most 16 (64 fp32 values to a thread), four where eight warps
// hold the row with them (14566 x 2048 with residual and 8-bit output: 45 us with
// four, 53 with two, 47 with eight, 56 with sixteen)
constexpr int NB_MAX = 16, NB_PREF = 4;

template <class T, bool VEC, bool NORM, bool Q8>
cudaError_t rows8_nb(int nb, int W, long long rows, int C, const RmsArgs& a, cudaStream_t s) {
  const long long grid = (rows + 8 / W - 1) / (8 / W);
  cudaError_t e;
  if (nb <= 1) e = launch_pdl(k_rows8<T, 1, VEC, NORM, Q8>, (unsigned)grid, 256, 0, s, rows, C, W, a);
  else if (nb <= 2) e = launch_pdl(k_rows8<T, 2, VEC, NORM, Q8>, (unsigned)grid, 256, 0, s, rows, C, W, a);
  else if (nb <= 3) e = launch_pdl(k_rows8<T, 3, VEC, NORM, Q8>, (unsigned)grid, 256, 0, s, rows, C, W, a);
  else if (nb <= 4) e = launch_pdl(k_rows8<T, 4, VEC, NORM, Q8>, (unsigned)grid, 256, 0, s, rows, C, W, a);
  else if (nb <= 8) e = launch_pdl(k_rows8<T, 8, VEC, NORM, Q8>, (unsigned)grid, 256, 0, s, rows, C, W, a);
  else e = launch_pdl(k_rows8<T, NB_MAX, VEC, NORM, Q8>, (unsigned)grid, 256, 0, s, rows, C, W, a);
  return e != cudaSuccess ? e : launched();
}

template <class T, bool NORM>
cudaError_t rows8(long long rows, int C, const RmsArgs& a, cudaStream_t s) {
  const int blocks = (C + 127) / 128;
  // Warps to a row: as few as hold it with NB_PREF blocks each, more while the rows
  // alone leave the SMs without 8 warps each.
  int W = 1;
  while (W < 8 && (blocks > NB_PREF * W || (rows * W < 152 * 8 && blocks > W))) W *= 2;
  const int nb = (blocks + W - 1) / W;
  if constexpr (NORM) {
    if (nb > NB_MAX) {
      // (the limit of the widest row, not of this one: it is the process's, and a narrower
      // row's call on another thread may come between it and the launch)
      const cudaError_t e = cudaFuncSetAttribute(k_rows8_wide<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, RMS_COLS_MAX * 4);
      if (e != cudaSuccess) return e;
      const cudaError_t l = launch_pdl(k_rows8_wide<T>, (unsigned)rows, 1024, (size_t)C * 4, s, C, a);
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
  if (tile == 1)   // wider rows than registers hold: runs of columns, each a matrix of its own
    return for_runs(C, 128 * 8 * NB_MAX, [&](long long c, long long n) {
      const Quant8Out part = {reinterpret_cast<uint8_t*>(o.q) + c, o.ldq, o.scale + c / 128 * o.lds, o.lds};
      return quant8<T>(1, rows, (int)n, reinterpret_cast<const T*>(x) + c, ldx, part, s);
    });
  // (row blocks in the grid's second dimension, at most 65535 to a launch)
  return for_runs(rows, 65535 * 128ll, [&](long long r, long long n) {
    const T* xr = reinterpret_cast<const T*>(x) + r * ldx;
    const Quant8Out part = {reinterpret_cast<uint8_t*>(o.q) + r * o.ldq, o.ldq, o.scale + (r / 128) * o.lds, o.lds};
    const dim3 grid((C + 127) / 128, (unsigned)((n + 127) / 128));
    const cudaError_t e = C % 4 == 0 && al4<T>(x, ldx) ? launch_pdl(k_quant8_tile<T, true>, grid, 256, 0, s, n, C, xr, ldx, part)
                                                       : launch_pdl(k_quant8_tile<T, false>, grid, 256, 0, s, n, C, xr, ldx, part);
    return e != cudaSuccess ? e : launched();
  });
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
