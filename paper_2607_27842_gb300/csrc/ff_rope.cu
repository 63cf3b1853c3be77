// Rotary positions with several axes on q and k, with the root-mean-square norm of
// each head in front of them where its weight is given (formula: featfix_op_rope).
// Bound by memory: q and k are read and written once; a row's sines and cosines are
// formed once for all of its heads.
#include "ff_common.cuh"

#include <algorithm>

namespace ff {

namespace {

// cos and sin of pos * freq turns.  The product's rounding error and the
// frequency's low part are added to the fraction of a turn that is left, so the
// angle keeps fp32 accuracy at large positions (pos is split: it may have more bits
// than a float).
__device__ __forceinline__ float2 turn(int pos, float2 f) {
  const float ph = (float)(pos & ~0xffff), pl = (float)(pos & 0xffff);
  const float th = ph * f.x, tl = pl * f.x;
  float t = (th - rintf(th)) + (tl - rintf(tl));
  t += __fmaf_rn(ph, f.x, -th) + __fmaf_rn(pl, f.x, -tl) + __fmaf_rn(ph, f.y, pl * f.y);
  t -= rintf(t);
  float s, c;
  sincospif(2.f * t, &s, &c);
  return make_float2(c, s);
}

// Eight elements of a head in one lane, as four fp32 pairs: columns 8 l .. 8 l + 7, or
// with halves and 8 l < rot columns 4 l .. 4 l + 3 of both halves.  Either way they
// are pairs 4 l .. 4 l + 3 where they are turned at all.
template <class T> struct Eight;
template <> struct Eight<float> {
  ulonglong2 r[2];
  __device__ __forceinline__ void load(const float* lo, const float* hi) {
    r[0] = *reinterpret_cast<const ulonglong2*>(lo);
    r[1] = *reinterpret_cast<const ulonglong2*>(hi);
  }
  __device__ __forceinline__ void get(f32x2 (&v)[4]) const { v[0] = r[0].x; v[1] = r[0].y; v[2] = r[1].x; v[3] = r[1].y; }
  static __device__ __forceinline__ void store(float* lo, float* hi, const f32x2 (&v)[4]) {
    *reinterpret_cast<ulonglong2*>(lo) = make_ulonglong2(v[0], v[1]);
    *reinterpret_cast<ulonglong2*>(hi) = make_ulonglong2(v[2], v[3]);
  }
};
template <> struct Eight<bf16> {
  uint2 r[2];
  __device__ __forceinline__ void load(const bf16* lo, const bf16* hi) {
    r[0] = *reinterpret_cast<const uint2*>(lo);
    r[1] = *reinterpret_cast<const uint2*>(hi);
  }
  __device__ __forceinline__ void get(f32x2 (&v)[4]) const {
    v[0] = bf2u(r[0].x); v[1] = bf2u(r[0].y); v[2] = bf2u(r[1].x); v[3] = bf2u(r[1].y);
  }
  static __device__ __forceinline__ void store(bf16* lo, bf16* hi, const f32x2 (&v)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 t = __floats2bfloat162_rn(lo_f(v[i]), hi_f(v[i]));
      w[i] = *reinterpret_cast<const uint32_t*>(&t);
    }
    *reinterpret_cast<uint2*>(lo) = make_uint2(w[0], w[1]);
    *reinterpret_cast<uint2*>(hi) = make_uint2(w[2], w[3]);
  }
};

constexpr int ROPE_ROWS = 8;   // most rows to a block

// R rows to a block, 2^lgl lanes to a head.  A group of lanes keeps its head (its
// addresses and the norm's weight) and goes down the rows, four at a time: hc heads
// lie side by side over the groups, and where that leaves groups over, `par` rows do.
// The first loads are under way while the block forms its sines and cosines.
// NORM: some side has a weight.  HALVES: pairs are half a width apart.
template <class T, bool NORM, bool HALVES>
__global__ void __launch_bounds__(256) k_rope(long long rows, int R, int lgl, int hc, int par,
                                              const __grid_constant__ RopeArgs a) {
  __shared__ __align__(16) float2 cs[ROPE_ROWS][ROPE_PAIRS];
  const int np = a.rot >> 1, hq = a.side[0].heads, H = hq + a.side[1].heads;
  const long long r0 = (long long)blockIdx.x * R;
  const int n = (int)min((long long)R, rows - r0);
  const int l = threadIdx.x & ((1 << lgl) - 1), grp = threadIdx.x >> lgl;
  const int first = grp / hc, h0 = grp - first * hc;   // the group's first row and head
  const bool turned = 8 * l < a.rot;
  // the lane's columns: first four, last four
  const int lo = HALVES && turned ? 4 * l : 8 * l, hi = HALVES && turned ? np + 4 * l : 8 * l + 4;
  pdl_trigger();
  pdl_wait();
  const float inv_hd = 1.f / (float)a.hd;
  bool made = false;
  for (int hb = blockIdx.y * hc; hb < H; hb += gridDim.y * hc) {   // (the same count of rounds for every thread, as below)
    const int head = hb + h0;
    const bool second = head >= hq, on = head < H && first < par && 8 * l < a.hd;
    const T* x = reinterpret_cast<const T*>(second ? a.side[1].x : a.side[0].x);
    T* o = reinterpret_cast<T*>(second ? a.side[1].out : a.side[0].out);
    const T* wt = reinterpret_cast<const T*>(second ? a.side[1].weight : a.side[0].weight);
    const long long ldx = second ? a.side[1].ldx : a.side[0].ldx, ldo = second ? a.side[1].ldo : a.side[0].ldo;
    const int col = (second ? head - hq : head) * a.hd;
    x += (r0 + first) * ldx + col;
    o += (r0 + first) * ldo + col;
    f32x2 w[4];
    if (NORM && wt && on) {
      Eight<T> e;
      e.load(wt + lo, wt + hi);
      e.get(w);
    }
    for (int rb = 0; rb < R; rb += 4 * par) {
      Eight<T> e[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (on && rb + i * par + first < n) e[i].load(x + (rb + i * par) * ldx + lo, x + (rb + i * par) * ldx + hi);
      if (!made) {
        for (int i = threadIdx.x; i < n * np; i += 256) {
          const int r = i / np, p = i - r * np;
          cs[r][p] = turn(a.pos[a.axis[p] * a.ld_pos + r0 + r], a.freq[p]);
        }
        __syncthreads();
        made = true;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = rb + i * par + first;
        const bool in = on && r < n;
        f32x2 v[4] = {0, 0, 0, 0};
        if (in) e[i].get(v);
        if (NORM) {   // (every lane of the warp takes part)
          const f32x2 s2 = ffma2(v[3], v[3], ffma2(v[2], v[2], ffma2(v[1], v[1], fmul2(v[0], v[0]))));
          float ss = lo_f(s2) + hi_f(s2);
          for (int k = 1; k < 1 << lgl; k <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, k);
          if (wt) {
            const float rstd = rsqrtf(fmaf(ss, inv_hd, a.eps));
            const f32x2 r2 = f2u(rstd, rstd);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = fmul2(fmul2(v[k], r2), w[k]);
          }
        }
        if (!in) continue;
        if (turned) {
          const float4* c4 = reinterpret_cast<const float4*>(&cs[r][4 * l]);
          const float4 c01 = c4[0], c23 = c4[1];
          // (single operations: building packed pairs of cosines costs more than they save)
          const float c[4] = {c01.x, c01.z, c23.x, c23.z}, s[4] = {c01.y, c01.w, c23.y, c23.w};
          if (HALVES) {   // v[0], v[1]: four of the first half, v[2], v[3]: of the second
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const float x0 = lo_f(v[k]), x1 = hi_f(v[k]), y0 = lo_f(v[k + 2]), y1 = hi_f(v[k + 2]);
              v[k] = f2u(x0 * c[2 * k] - y0 * s[2 * k], x1 * c[2 * k + 1] - y1 * s[2 * k + 1]);
              v[k + 2] = f2u(x0 * s[2 * k] + y0 * c[2 * k], x1 * s[2 * k + 1] + y1 * c[2 * k + 1]);
            }
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float x = lo_f(v[k]), y = hi_f(v[k]);
              v[k] = f2u(x * c[k] - y * s[k], x * s[k] + y * c[k]);
            }
          }
        }
        Eight<T>::store(o + (rb + i * par) * ldo + lo, o + (rb + i * par) * ldo + hi, v);
      }
    }
  }
}

// Any head width, stride and alignment: one block to a row, a warp to a head, the head
// in shared memory.
template <class T>
__global__ void __launch_bounds__(256) k_rope_any(const __grid_constant__ RopeArgs a) {
  __shared__ float2 cs[ROPE_PAIRS];
  __shared__ float buf[8][2 * ROPE_PAIRS];
  const long long r = blockIdx.x;
  const int np = a.rot >> 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_trigger();
  pdl_wait();
  for (int p = threadIdx.x; p < np; p += 256) cs[p] = turn(a.pos[a.axis[p] * a.ld_pos + r], a.freq[p]);
  __syncthreads();
  for (int h = warp; h < a.side[0].heads + a.side[1].heads; h += 8) {
    const RopeSide& sd = a.side[h < a.side[0].heads ? 0 : 1];
    const long long at = (long long)(h < a.side[0].heads ? h : h - a.side[0].heads) * a.hd;
    const T* x = reinterpret_cast<const T*>(sd.x) + r * sd.ldx + at;
    T* o = reinterpret_cast<T*>(sd.out) + r * sd.ldo + at;
    const T* w = reinterpret_cast<const T*>(sd.weight);
    float ss = 0.f;
    for (int c = lane; c < a.hd; c += 32) {
      const float v = to_f(x[c]);
      buf[warp][c] = v;
      ss = fmaf(v, v, ss);
    }
    if (w) {
#pragma unroll
      for (int k = 16; k; k >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, k);
      const float rstd = rsqrtf(ss / (float)a.hd + a.eps);
      for (int c = lane; c < a.hd; c += 32) buf[warp][c] *= rstd * to_f(w[c]);
    }
    __syncwarp();
    for (int p = lane; p < np; p += 32) {
      const int i = a.halves ? p : 2 * p, j = a.halves ? p + np : 2 * p + 1;
      const float u = buf[warp][i], v = buf[warp][j];
      o[i] = from_f<T>(u * cs[p].x - v * cs[p].y);
      o[j] = from_f<T>(u * cs[p].y + v * cs[p].x);
    }
    for (int c = a.rot + lane; c < a.hd; c += 32) o[c] = from_f<T>(buf[warp][c]);
    __syncwarp();
  }
}

template <class T>
cudaError_t rope(long long rows, const RopeArgs& a, cudaStream_t s) {
  // four-element vectors: rows, heads and both halves on their boundary
  bool vec = a.hd % 8 == 0 && a.rot % 8 == 0;
  for (const RopeSide& sd : a.side)
    if (sd.heads)
      vec = vec && sd.ldx % 4 == 0 && sd.ldo % 4 == 0 &&
            !(((uintptr_t)sd.x | (uintptr_t)sd.out | (uintptr_t)sd.weight) & (4 * sizeof(T) - 1));
  if (!vec) {
    const cudaError_t e = launch_pdl(k_rope_any<T>, (unsigned)rows, 256, 0, s, a);
    return e != cudaSuccess ? e : launched();
  }
  int lgl = 0;
  while (8 << lgl < a.hd) ++lgl;
  const int H = a.side[0].heads + a.side[1].heads, groups = 256 >> lgl;
  // even rounds over the heads; rows side by side where the heads leave groups over;
  // four rows at a time to a group, fewer where the rows would not fill the SMs
  const int rounds = (H + groups - 1) / groups, hc = (H + rounds - 1) / rounds;
  const int par = std::min(ROPE_ROWS, groups / hc);
  int R = std::min(ROPE_ROWS, 4 * par);
  while (R > par && (rows + R - 1) / R < 2 * 152) R = std::max(par, R / 2);
  const long long grid = (rows + R - 1) / R;
  // few rows: the rounds over the heads are blocks of their own
  const dim3 grid2((unsigned)grid, grid < 152 ? rounds : 1);
  const bool norm = a.side[0].weight || a.side[1].weight;
  auto fn = norm ? (a.halves ? k_rope<T, true, true> : k_rope<T, true, false>)
                 : (a.halves ? k_rope<T, false, true> : k_rope<T, false, false>);
  const cudaError_t e = launch_pdl(fn, grid2, 256, 0, s, rows, R, lgl, hc, par, a);
  return e != cudaSuccess ? e : launched();
}

}  // namespace

cudaError_t launch_rope(DType dt, long long rows, const RopeArgs& a, cudaStream_t s) {
  if (rows <= 0) return cudaSuccess;
  return dt == F32 ? rope<float>(rows, a, s) : rope<bf16>(rows, a, s);
}

}  // namespace ff
