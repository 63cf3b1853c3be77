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

// Eight elements of a head in one lane: columns 8 l .. 8 l + 7, or with halves and
// 8 l < rot columns 4 l .. 4 l + 3 of both halves.  Either way they are pairs 4 l ..
// 4 l + 3 where they are turned at all.
template <class T> struct Eight;
template <> struct Eight<float> {
  float4 r[2];
  __device__ __forceinline__ void load(const float* lo, const float* hi) {
    r[0] = *reinterpret_cast<const float4*>(lo);
    r[1] = *reinterpret_cast<const float4*>(hi);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = r[0].x; v[1] = r[0].y; v[2] = r[0].z; v[3] = r[0].w;
    v[4] = r[1].x; v[5] = r[1].y; v[6] = r[1].z; v[7] = r[1].w;
  }
  static __device__ __forceinline__ void store(float* lo, float* hi, const float (&v)[8]) {
    *reinterpret_cast<float4*>(lo) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(hi) = make_float4(v[4], v[5], v[6], v[7]);
  }
};
template <> struct Eight<bf16> {
  uint2 r[2];
  __device__ __forceinline__ void load(const bf16* lo, const bf16* hi) {
    r[0] = *reinterpret_cast<const uint2*>(lo);
    r[1] = *reinterpret_cast<const uint2*>(hi);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    unpack16(make_uint4(r[0].x, r[0].y, r[1].x, r[1].y), v);
  }
  static __device__ __forceinline__ void store(bf16* lo, bf16* hi, const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const __nv_bfloat162 a = __floats2bfloat162_rn(v[4 * i], v[4 * i + 1]), b = __floats2bfloat162_rn(v[4 * i + 2], v[4 * i + 3]);
      *reinterpret_cast<uint2*>(i ? hi : lo) =
          make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
    }
  }
};

constexpr int ROPE_ROWS = 8;   // most rows to a block

// R rows to a block.  A group of 2^lgl lanes takes a head, four heads at a time (their
// loads come first, the block's first ones before its sines and cosines).
template <class T>
__global__ void __launch_bounds__(256) k_rope(long long rows, int R, int lgl, const __grid_constant__ RopeArgs a) {
  __shared__ __align__(16) float2 cs[ROPE_ROWS][ROPE_PAIRS];
  const int np = a.rot >> 1, H = a.side[0].heads + a.side[1].heads;
  const long long r0 = (long long)blockIdx.x * R;
  const int n = (int)min((long long)R, rows - r0), units = n * H;
  const int l = threadIdx.x & ((1 << lgl) - 1), groups = 256 >> lgl;
  const bool on = 8 * l < a.hd, turned = 8 * l < a.rot;
  // the lane's columns: first four, last four
  const int lo = a.halves && turned ? 4 * l : 8 * l, hi = a.halves && turned ? np + 4 * l : 8 * l + 4;
  pdl_trigger();
  pdl_wait();
  for (int base = threadIdx.x >> lgl; base - (int)(threadIdx.x >> lgl) < units; base += 4 * groups) {
    Eight<T> e[4];
    int row[4], head[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int u = base + i * groups;
      row[i] = u < units ? u / H : -1;
      head[i] = u - row[i] * H;
      if (row[i] < 0 || !on) continue;
      const RopeSide& sd = a.side[head[i] < a.side[0].heads ? 0 : 1];
      const T* x = reinterpret_cast<const T*>(sd.x) + (r0 + row[i]) * sd.ldx +
                   (head[i] < a.side[0].heads ? head[i] : head[i] - a.side[0].heads) * a.hd;
      e[i].load(x + lo, x + hi);
    }
    if (base < groups) {   // (every thread's first time round)
      for (int i = threadIdx.x; i < n * np; i += 256) {
        const int r = i / np, p = i - r * np;
        cs[r][p] = turn(a.pos[a.axis[p] * a.ld_pos + r0 + r], a.freq[p]);
      }
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool in = row[i] >= 0 && on;
      const bool second = head[i] >= a.side[0].heads;
      float v[8] = {};
      if (in) e[i].get(v);
      const RopeSide& sd = a.side[second ? 1 : 0];
      // (one side may have a norm and the other none: every lane of the warp takes part)
      if (a.side[0].weight || a.side[1].weight) {
        float ss = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) ss = fmaf(v[k], v[k], ss);
        for (int o = 1; o < 1 << lgl; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        if (sd.weight && in) {
          const T* wt = reinterpret_cast<const T*>(sd.weight);
          Eight<T> we;
          we.load(wt + lo, wt + hi);
          float w[8];
          we.get(w);
          const float rstd = rsqrtf(ss / (float)a.hd + a.eps);
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] *= rstd * w[k];
        }
      }
      if (!in) continue;
      if (turned) {
        const float4* c4 = reinterpret_cast<const float4*>(&cs[row[i]][4 * l]);
        const float4 c01 = c4[0], c23 = c4[1];
        const float c[4] = {c01.x, c01.z, c23.x, c23.z}, s[4] = {c01.y, c01.w, c23.y, c23.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (a.halves) {   // (two branches, so that every index is known to the compiler)
            const float x = v[k], y = v[k + 4];
            v[k] = x * c[k] - y * s[k];
            v[k + 4] = x * s[k] + y * c[k];
          } else {
            const float x = v[2 * k], y = v[2 * k + 1];
            v[2 * k] = x * c[k] - y * s[k];
            v[2 * k + 1] = x * s[k] + y * c[k];
          }
        }
      }
      T* o = reinterpret_cast<T*>(sd.out) + (r0 + row[i]) * sd.ldo + (second ? head[i] - a.side[0].heads : head[i]) * a.hd;
      Eight<T>::store(o + lo, o + hi, v);
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
  // about four heads to a group of lanes, so all of a block's loads are under way at once
  const int H = a.side[0].heads + a.side[1].heads, groups = 256 >> lgl;
  const int R = std::max(1, std::min(ROPE_ROWS, 4 * groups / H));
  const long long grid = (rows + R - 1) / R;
  const cudaError_t e = launch_pdl(k_rope<T>, (unsigned)grid, 256, 0, s, rows, R, lgl, a);
  return e != cudaSuccess ? e : launched();
}

}  // namespace

cudaError_t launch_rope(DType dt, long long rows, const RopeArgs& a, cudaStream_t s) {
  if (rows <= 0) return cudaSuccess;
  return dt == F32 ? rope<float>(rows, a, s) : rope<bf16>(rows, a, s);
}

}  // namespace ff
