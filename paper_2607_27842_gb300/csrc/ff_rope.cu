// Rotary positions with several axes on q and k, with the root-mean-square norm of
// each head in front of them where its weight is given (formula: featfix_op_rope).
// Bound by memory without the norm (14566 rows of 16 + 16 heads of 128, bf16: 39.2 us, 6.1
// TB/s), by shuffles and issue with it (44.6 us, 5.4 TB/s): q and k are read and written
// once; a row's sines and cosines are formed once for all of its heads.
#include "ff_common.cuh"
#include "ff_q8.cuh"

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
  __device__ __forceinline__ void load(const float* lo, const float* hi, int, int) {
    r[0] = *reinterpret_cast<const ulonglong2*>(lo);
    r[1] = *reinterpret_cast<const ulonglong2*>(hi);
  }
  __device__ __forceinline__ void get(f32x2 (&v)[4]) const { v[0] = r[0].x; v[1] = r[0].y; v[2] = r[1].x; v[3] = r[1].y; }
  static __device__ __forceinline__ void store(float* lo, float* hi, int, int, const f32x2 (&v)[4]) {
    *reinterpret_cast<ulonglong2*>(lo) = make_ulonglong2(v[0], v[1]);
    *reinterpret_cast<ulonglong2*>(hi) = make_ulonglong2(v[2], v[3]);
  }
};
template <> struct Eight<bf16> {
  uint2 r[2];
  __device__ __forceinline__ void load(const bf16* lo, const bf16* hi, int, int) {
    r[0] = *reinterpret_cast<const uint2*>(lo);
    r[1] = *reinterpret_cast<const uint2*>(hi);
  }
  __device__ __forceinline__ void get(f32x2 (&v)[4]) const {
    v[0] = bf2u(r[0].x); v[1] = bf2u(r[0].y); v[2] = bf2u(r[1].x); v[3] = bf2u(r[1].y);
  }
  static __device__ __forceinline__ void store(bf16* lo, bf16* hi, int, int, const f32x2 (&v)[4]) {
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

// The same element by element, nlo and nhi of each four: any alignment, pairs and heads
// that end inside a lane's share.
template <class T> struct EightAny {
  T r[8];
  __device__ __forceinline__ void load(const T* lo, const T* hi, int nlo, int nhi) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      r[k] = k < nlo ? lo[k] : from_f<T>(0.f);
      r[4 + k] = k < nhi ? hi[k] : from_f<T>(0.f);
    }
  }
  __device__ __forceinline__ void get(f32x2 (&v)[4]) const {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = f2u(to_f(r[2 * k]), to_f(r[2 * k + 1]));
  }
  static __device__ __forceinline__ void store(T* lo, T* hi, int nlo, int nhi, const f32x2 (&v)[4]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (k < nlo) lo[k] = from_f<T>(k & 1 ? hi_f(v[k / 2]) : lo_f(v[k / 2]));
      if (k < nhi) hi[k] = from_f<T>(k & 1 ? hi_f(v[2 + k / 2]) : lo_f(v[2 + k / 2]));
    }
  }
};

template <bool C, class A, class B> struct Pick { using type = A; };
template <class A, class B> struct Pick<false, A, B> { using type = B; };

constexpr int ROPE_ROWS = 8;   // most rows to a block

// How a head's pairs lie: neighbours whose axes fill whole lanes; neighbours, and the axes
// end inside a lane's four; half a width apart.
enum Form { PAIRS, PAIRS_TAIL, HALVES };

// Turns (and norms) a group of lanes' share of one side's heads of one row: heads g, g +
// step, .., four at a time, their loads in front.  c, s: the lane's four cosines and
// sines.  np: all pairs of a head; PAIRS_TAIL keeps what lies behind them as it is (an
// infinity there would make its neighbour NaN, times a sine of zero).  A form of its own:
// with the choice 14566 rows of 16 + 16 heads of 128, 74 columns turned, take 44.3 us with
// norm instead of 41.9, and all 128 turned would take 46.6 instead of 44.6.
template <class T, class E, bool NORM, Form FORM, class Make>
__device__ __forceinline__ void rope_side(const RopeSide& sd, long long r, int g, int step, int l, int lanes, int lo, int hi,
                                          int nlo, int nhi, bool on, bool turned, int np, int hd, float inv_hd, float eps, float (&c)[4], float (&s)[4],
                                          const float2* cs, bool& made, const Make& make) {
  const T* x = reinterpret_cast<const T*>(sd.x) + r * sd.ldx;
  T* o = reinterpret_cast<T*>(sd.out) + r * sd.ldo;
  const T* wt = reinterpret_cast<const T*>(sd.weight);
  f32x2 w[4];
  if (NORM && wt && on) {
    E e;
    e.load(wt + lo, wt + hi, nlo, nhi);
    e.get(w);
  }
  for (int h0 = 0; h0 < sd.heads; h0 += 4 * step) {   // (the same count of rounds for every lane)
    E e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int h = h0 + i * step + g;
      if (on && h < sd.heads) e[i].load(x + h * hd + lo, x + h * hd + hi, nlo, nhi);
    }
    if (!made) {   // the block's sines and cosines; this lane's
      make();
      __syncthreads();
      made = true;
      if (on && turned) {
        const float4 c01 = reinterpret_cast<const float4*>(cs + 4 * l)[0], c23 = reinterpret_cast<const float4*>(cs + 4 * l)[1];
        c[0] = c01.x; c[1] = c01.z; c[2] = c23.x; c[3] = c23.z;
        s[0] = c01.y; s[1] = c01.w; s[2] = c23.y; s[3] = c23.w;
      }
    }
    float rs[4];
    if (NORM && wt) {
      // Four sums over the group's lanes at once: the first two steps also halve the sums
      // a lane holds, so lane l ends with that of head l % 4, and forms one root
      // for it (9 shuffles and one root where each sum alone takes 16 and four)
      float q[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x2 v[4] = {0, 0, 0, 0};
        if (on && h0 + i * step + g < sd.heads) e[i].get(v);
        const f32x2 s2 = ffma2(v[3], v[3], ffma2(v[2], v[2], ffma2(v[1], v[1], fmul2(v[0], v[0]))));
        q[i] = lo_f(s2) + hi_f(s2);
      }
      const bool b0 = l & 1, b1 = l & 2;
      const float p0 = (b0 ? q[1] : q[0]) + __shfl_xor_sync(0xffffffffu, b0 ? q[0] : q[1], 1);
      const float p1 = (b0 ? q[3] : q[2]) + __shfl_xor_sync(0xffffffffu, b0 ? q[2] : q[3], 1);
      float ss = (b1 ? p1 : p0) + __shfl_xor_sync(0xffffffffu, b1 ? p0 : p1, 2);
      for (int k = 4; k < lanes; k <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, k);
      const float rstd = rsqrtf(fmaf(ss, inv_hd, eps));
#pragma unroll
      for (int i = 0; i < 4; ++i) rs[i] = __shfl_sync(0xffffffffu, rstd, i, 4);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int h = h0 + i * step + g;
      if (!on || h >= sd.heads) continue;
      f32x2 v[4];
      e[i].get(v);
      if (NORM && wt) {
        const f32x2 r2 = f2u(rs[i], rs[i]);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = fmul2(fmul2(v[k], r2), w[k]);
      }
      if (turned) {
        // (single operations: building packed pairs of cosines costs more than they save)
        if (FORM == HALVES) {   // v[0], v[1]: four of the first half, v[2], v[3]: of the second
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float x0 = lo_f(v[k]), x1 = hi_f(v[k]), y0 = lo_f(v[k + 2]), y1 = hi_f(v[k + 2]);
            v[k] = f2u(x0 * c[2 * k] - y0 * s[2 * k], x1 * c[2 * k + 1] - y1 * s[2 * k + 1]);
            v[k + 2] = f2u(x0 * s[2 * k] + y0 * c[2 * k], x1 * s[2 * k + 1] + y1 * c[2 * k + 1]);
          }
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float x0 = lo_f(v[k]), y0 = hi_f(v[k]);
            const f32x2 t = f2u(x0 * c[k] - y0 * s[k], x0 * s[k] + y0 * c[k]);
            v[k] = FORM == PAIRS || 4 * l + k < np ? t : v[k];
          }
        }
      }
      E::store(o + h * hd + lo, o + h * hd + hi, nlo, nhi, v);
    }
  }
}

// R rows to a block, 2^lgl lanes to a head; a group of lanes stays with one row (its
// sines and cosines in registers) and takes every step-th head of it, step = groups / R.
// The first loads are under way while the block forms its sines and cosines.
// NORM: some side has a weight.  bf16: at most 64
// registers, four blocks to an SM (14566 rows with norm 49.9 -> 44.7 us; five 50.5).
// ANY: rows of any alignment and pairs that end inside a lane's four, element by element.
template <class T, bool NORM, Form FORM, bool ANY>
__global__ void __launch_bounds__(256, sizeof(T) == 2 && !ANY ? 4 : 2)
    k_rope(long long rows, int lgr, int lgl, const __grid_constant__ RopeArgs a) {
  using E = typename Pick<ANY, EightAny<T>, Eight<T>>::type;
  __shared__ __align__(16) float2 cs[ROPE_ROWS][ROPE_PAIRS];
  const int np = a.rot >> 1, R = 1 << lgr;
  const long long r0 = (long long)blockIdx.x << lgr;
  const int n = (int)min((long long)R, rows - r0);
  const int l = threadIdx.x & ((1 << lgl) - 1), grp = threadIdx.x >> lgl;
  const int step = 256 >> (lgl + lgr), row = grp / step, g = grp & (step - 1);   // (a warp's groups: heads side by side)
  // the lane's columns of a head: first four and last four, and how many of each there are
  const bool turned = FORM == HALVES ? 4 * l < np : 8 * l < a.rot;
  int lo = 8 * l, hi = 8 * l + 4, nlo = 4, nhi = 4;
  if (FORM == HALVES && turned) {
    lo = 4 * l;
    hi = np + 4 * l;
    if (ANY) nlo = nhi = min(4, np - 4 * l);
  } else if (ANY) {
    if (FORM == HALVES) lo = a.rot + 8 * (l - ((np + 3) >> 2));
    hi = lo + 4;
    nlo = max(0, min(4, a.hd - lo));
    nhi = max(0, min(4, a.hd - hi));
  }
  const bool on = row < n && (ANY ? nlo > 0 : 8 * l < a.hd);
  const float inv_hd = 1.f / (float)a.hd;
  float c[4] = {}, s[4] = {};
  bool made = false;
  pdl_trigger();
  pdl_wait();
  auto make = [&] {
    const int up = (np + 3) & ~3;   // (whole fours: a lane reads its four at once)
    for (int i = threadIdx.x; i < n * up; i += 256) {
      const int r = i / up, p = i - r * up;
      cs[r][p] = p < np ? turn(a.pos[a.axis[p] * a.ld_pos + r0 + r], a.freq[p]) : make_float2(1.f, 0.f);
    }
  };
  rope_side<T, E, NORM, FORM>(a.side[0], r0 + row, g, step, l, 1 << lgl, lo, hi, nlo, nhi, on, turned, np, a.hd, inv_hd, a.eps, c, s, cs[row], made, make);
  rope_side<T, E, NORM, FORM>(a.side[1], r0 + row, g, step, l, 1 << lgl, lo, hi, nlo, nhi, on, turned, np, a.hd, inv_hd, a.eps, c, s, cs[row], made, make);
}

// Halves with columns behind them that together need more than 32 lanes (head widths of 250
// and up): R rows to a block, a warp to a head, a lane
// to every 32nd pair and every 32nd column that is not turned. 
template <class T>
__global__ void __launch_bounds__(256) k_rope_any(long long rows, int R, const __grid_constant__ RopeArgs a) {
  __shared__ float2 cs[ROPE_ROWS][ROPE_PAIRS];
  const long long r0 = (long long)blockIdx.x * R;
  const int n = (int)min((long long)R, rows - r0);
  const int np = a.rot >> 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int hq = a.side[0].heads, H = hq + a.side[1].heads;
  const float inv_hd = 1.f / (float)a.hd;
  pdl_trigger();
  pdl_wait();
  for (int i = threadIdx.x; i < n * np; i += 256) {
    const int k = i / np, p = i - k * np;
    cs[k][p] = turn(a.pos[a.axis[p] * a.ld_pos + r0 + k], a.freq[p]);
  }
  __syncthreads();
  for (int unit = warp; unit < n * H; unit += 8) {
    const int row = unit / H, h = unit - row * H;
    const long long r = r0 + row;
    const bool second = h >= hq;
    const long long at = (long long)(second ? h - hq : h) * a.hd;
    const T* x = reinterpret_cast<const T*>(second ? a.side[1].x : a.side[0].x) + r * (second ? a.side[1].ldx : a.side[0].ldx) + at;
    T* o = reinterpret_cast<T*>(second ? a.side[1].out : a.side[0].out) + r * (second ? a.side[1].ldo : a.side[0].ldo) + at;
    const T* w = reinterpret_cast<const T*>(second ? a.side[1].weight : a.side[0].weight);
    const T* x1 = x + (a.halves ? np : 1);   // a pair's second column
    const int ps = a.halves ? 1 : 2, rest = a.hd - a.rot;
    float u[4], v[4], t[8], ss = 0.f;   // pairs, columns past rot
    // (the loops end, for the whole warp, with the last column)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (32 * i >= np) break;
      const int p = lane + 32 * i;
      u[i] = p < np ? to_f(x[ps * p]) : 0.f;
      v[i] = p < np ? to_f(x1[ps * p]) : 0.f;
      ss = fmaf(u[i], u[i], fmaf(v[i], v[i], ss));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (32 * i >= rest) break;
      t[i] = lane + 32 * i < rest ? to_f(x[a.rot + lane + 32 * i]) : 0.f;
      ss = fmaf(t[i], t[i], ss);
    }
    if (w) {
#pragma unroll
      for (int k = 16; k; k >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, k);
      const float rstd = rsqrtf(fmaf(ss, inv_hd, a.eps));
      const T* w1 = w + (a.halves ? np : 1);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (32 * i >= np) break;
        const int p = min(lane + 32 * i, np - 1);
        u[i] *= rstd * to_f(w[ps * p]);
        v[i] *= rstd * to_f(w1[ps * p]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (32 * i >= rest) break;
        t[i] *= rstd * to_f(w[min(a.rot + lane + 32 * i, a.hd - 1)]);
      }
    }
    T* o1 = o + (a.halves ? np : 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (32 * i >= np) break;
      const int p = lane + 32 * i;
      if (p < np) {
        const float2 c = cs[row][p];
        o[ps * p] = from_f<T>(u[i] * c.x - v[i] * c.y);
        o1[ps * p] = from_f<T>(u[i] * c.y + v[i] * c.x);
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (32 * i >= rest) break;
      if (lane + 32 * i < rest) o[a.rot + lane + 32 * i] = from_f<T>(t[i]);
    }
  }
}

template <class T>
cudaError_t rope(long long rows, const RopeArgs& a, cudaStream_t s) {
  // four-element vectors: rows, heads and both halves on their boundary
  bool vec = a.hd % 8 == 0 && (!a.halves || a.rot % 8 == 0);
  for (const RopeSide& sd : a.side)
    if (sd.heads)
      vec = vec && sd.ldx % 4 == 0 && sd.ldo % 4 == 0 &&
            !(((uintptr_t)sd.x | (uintptr_t)sd.out | (uintptr_t)sd.weight) & (4 * sizeof(T) - 1));
  // lanes to a head: eight columns each, halves that are not whole vectors with lanes of
  // their own for the columns behind them; four at least
  const int lanes = a.halves && !vec ? (a.rot / 2 + 3) / 4 + (a.hd - a.rot + 7) / 8 : (a.hd + 7) / 8;
  if (lanes > 32) {
    int R = ROPE_ROWS;
    while (R > 1 && rows / R < 4 * 152) R /= 2;
    const cudaError_t e = launch_pdl(k_rope_any<T>, (unsigned)((rows + R - 1) / R), 256, 0, s, rows, R, a);
    return e != cudaSuccess ? e : launched();
  }
  int lgl = 2, lgr = 0;
  while (1 << lgl < lanes) ++lgl;
  // rows to a block: as many as leave a group of lanes four heads of the larger side at
  // a time, fewer where the rows would not fill the SMs twice
  const int heads = std::max(a.side[0].heads, a.side[1].heads), groups = 256 >> lgl;
  while ((2 << lgr) <= std::min(ROPE_ROWS, groups) && (groups >> lgr) * 4 > heads && rows >> (lgr + 1) >= 2 * 152) ++lgr;
  const long long grid = (rows + (1 << lgr) - 1) >> lgr;
  const bool norm = a.side[0].weight || a.side[1].weight;
  using Fn = decltype(&k_rope<T, false, PAIRS, false>);
  static const Fn fns[2][2][3] = {   // [norm][any][form]
      {{k_rope<T, false, PAIRS, false>, k_rope<T, false, PAIRS_TAIL, false>, k_rope<T, false, HALVES, false>},
       {nullptr, k_rope<T, false, PAIRS_TAIL, true>, k_rope<T, false, HALVES, true>}},
      {{k_rope<T, true, PAIRS, false>, k_rope<T, true, PAIRS_TAIL, false>, k_rope<T, true, HALVES, false>},
       {nullptr, k_rope<T, true, PAIRS_TAIL, true>, k_rope<T, true, HALVES, true>}}};
  const Fn fn = fns[norm][!vec][a.halves ? HALVES : vec && a.rot % 8 == 0 ? PAIRS : PAIRS_TAIL];
  const cudaError_t e = launch_pdl(fn, (unsigned)grid, 256, 0, s, rows, lgr, lgl, a);
  return e != cudaSuccess ? e : launched();
}

}  // namespace

cudaError_t launch_rope(DType dt, long long rows, const RopeArgs& a, cudaStream_t s) {
  if (rows <= 0) return cudaSuccess;
  return dt == F32 ? rope<float>(rows, a, s) : rope<bf16>(rows, a, s);
}

}  // namespace ff
