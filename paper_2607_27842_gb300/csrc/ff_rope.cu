// Rotary positions with several axes on q and k, with the root-mean-square
// norm of each head in front of them where its weight is given.
#include "ff_common.cuh"

namespace ff {

namespace {

// cos and sin of pos * freq turns.  The product's rounding error and the
// frequency's low part are added to the fraction of a turn that is left, so the
// angle keeps fp32 accuracy at every int32 position (pos is split: it may have more
// bits than a float).
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

// One block per row, a warp per head.
template <class T>
__global__ void __launch_bounds__(256) k_rope(const __grid_constant__ RopeArgs a) {
  __shared__ float2 cs[ROPE_PAIRS];
  __shared__ float buf[8][2 * ROPE_PAIRS];
  const long long r = blockIdx.x;
  const int np = a.rot >> 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
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

}  // namespace

cudaError_t launch_rope(DType dt, long long rows, const RopeArgs& a, cudaStream_t s) {
  if (rows <= 0) return cudaSuccess;
  if (dt == F32)
    k_rope<float><<<(unsigned)rows, 256, 0, s>>>(a);
  else
    k_rope<bf16><<<(unsigned)rows, 256, 0, s>>>(a);
  return launched();
}

}  // namespace ff
