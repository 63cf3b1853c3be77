// The norms at the end of a block and at the beginning of the next one, with gate and
// residual between them (formulas: featfix_op_block_norms).  Bound by memory: x and y are read
// once into registers, and what is written is computed from there.
#include "ff_host.h"
#include "ff_kv8.cuh"
#include "ff_rows8.cuh"

#include <algorithm>

namespace ff {

namespace {

// Rows of all warps of a row slot meet in shared memory at a barrier of their own.
__device__ __forceinline__ void slot_sync(int slot, int warps) {
  asm volatile("bar.sync %0, %1;" ::"r"(slot + 1), "r"(32 * warps) : "memory");
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Eight adjacent columns of a lane, as they are in memory and as four fp32 pairs.
template <class T> struct Cols {
  uint4 r[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r[i] = make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void get(f32x2 (&v)[4]) const {
    if constexpr (sizeof(T) == 2) {
      v[0] = bf2u(r[0].x), v[1] = bf2u(r[0].y), v[2] = bf2u(r[0].z), v[3] = bf2u(r[0].w);
    } else {
      const ulonglong2 a = *reinterpret_cast<const ulonglong2*>(&r[0]), b = *reinterpret_cast<const ulonglong2*>(&r[1]);
      v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
    }
  }
  static __device__ __forceinline__ void store(T* p, const f32x2 (&v)[4]) {
    if constexpr (sizeof(T) == 2) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(lo_f(v[i]), hi_f(v[i]));
        w[i] = *reinterpret_cast<const uint32_t*>(&b);
      }
      *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      reinterpret_cast<ulonglong2*>(p)[0] = make_ulonglong2(v[0], v[1]);
      reinterpret_cast<ulonglong2*>(p)[1] = make_ulonglong2(v[2], v[3]);
    }
  }
};

// Rows of whole 16-byte vectors: W warps to a row (1, 2, 4 or 8; eight warps to a block), NB adjacent pieces of
// 256 columns to a warp, eight adjacent columns to a lane.  A block goes over rows of one sample,
// the next row's loads under way meanwhile.  Weights and modulation enter as three factors of a
// column, h = resid_scale x + p norm(y), z = q norm(h) + s, from shared memory: read from L2 for every
// row they are three times the bytes of x and y, and in registers (48 for 512 columns) they leave 16 warps
// to an SM, which do not hide the two norms' latencies (14566 x 2048: 99 us).  Now 36 us there with modulation and
// 8-bit output, 5.8 TB/s, where warps wait for shared memory and for each other's sums; 4000 x 8192 51 us; fp32 85 us.
//
// Blocks to an SM: as many as leave a lane the registers for its pieces of the two rows.  In fp32 three blocks
// of two pieces (80 registers, 130 bytes spilled) take 89.5 us for 14566 x 2048 and 188 for x 4096, two 85 and 151;
// two of four pieces (350 bytes spilled) 130 for 4000 x 8192, one 91.
template <class T, int NB> constexpr int NORMS_BLOCKS = NB * (int)sizeof(T) <= 4 ? 3 : NB * (int)sizeof(T) <= 12 ? 2 : 1;
template <class T, int NB, bool Q8>
__global__ void __launch_bounds__(256, NORMS_BLOCKS<T, NB>)
    k_block_norms(long long rows, int C, int W, long long per, int chunks, const __grid_constant__ BlockNormsArgs a) {
  extern __shared__ __align__(16) float factors[];   // p, q, s: pieces of two halves, a lane's four columns each
  __shared__ __align__(16) float sums[2][2][64];   // of a slot's warps (8 places to a slot, 0 where it has fewer): squares, means
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, w = warp & (W - 1), slot = warp / W, slots = 8 / W;
  const int c0 = w * NB * 256 + 8 * lane;
  const int wide = W * NB * 256;   // columns of the lanes
  const bool ragged = C != wide;   // some lanes have pieces behind the row's end
  // (sample, chunk of its rows) of this block
  const long long sample = blockIdx.x / chunks, first = sample * a.rpb + (blockIdx.x - sample * chunks) * per;
  const long long end = min(rows, min((sample + 1) * a.rpb, first + per));
  float *fp = factors, *fq = fp + wide, *fs = fq + wide;
  const bool has_s = a.shift != nullptr;
  bool in[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) in[i] = c0 + 256 * i < C;
  pdl_trigger();
  pdl_wait();

  const T* y = reinterpret_cast<const T*>(a.y) + (first + slot) * a.ldy + c0;   // of the next row to load
  const T* x = reinterpret_cast<const T*>(a.x) + (first + slot) * a.ldx + c0;
  const long long step_y = a.ldy * slots, step_x = a.ldx * slots;
  Cols<T> fy[NB], fx[NB];
  auto load_row = [&] {
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      if (in[i]) fy[i].load(y + 256 * i);
      if (in[i] && a.x) fx[i].load(x + 256 * i);
    }
    y += step_y;
    x += step_x;
  };
#pragma unroll
  for (int i = 0; i < NB; ++i) fy[i].zero(), fx[i].zero();
  if (first + slot < end) load_row();
  // Factors of eight adjacent columns at a time: every load of them is under way before the first is used
  // (column by column 4000 x 8192 took 62 us, 51 so).
  auto eight = [&](const float* m, float (&v)[8]) {
    if (!((uintptr_t)m & 15)) {
      const float4 l = reinterpret_cast<const float4*>(m)[0], h = reinterpret_cast<const float4*>(m)[1];
      v[0] = l.x, v[1] = l.y, v[2] = l.z, v[3] = l.w, v[4] = h.x, v[5] = h.y, v[6] = h.z, v[7] = h.w;
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = m[k];
    }
  };
  auto eight_of = [&](const void* m, int c, Cols<T>& v) {
    const T* p = reinterpret_cast<const T*>(m) + c;
    if (!((uintptr_t)p & 15)) {
      v.load(p);
    } else {
      __align__(16) T e[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) e[k] = p[k];
#pragma unroll
      for (int k = 0; k < (int)sizeof(T) / 2; ++k) v.r[k] = reinterpret_cast<const uint4*>(e)[k];
    }
  };
  for (int c = 8 * threadIdx.x; c < wide; c += 2048) {
    const bool there = c < C;
    float g[8], sc[8], sh[8];
    Cols<T> wa, wb;
#pragma unroll
    for (int k = 0; k < 8; ++k) g[k] = 1.f, sc[k] = sh[k] = 0.f;
    if (a.gate && there) eight(a.gate + sample * a.gate_stride + c, g);
    if (a.scale && there) eight(a.scale + sample * a.scale_stride + c, sc);
    if (has_s && there) eight(a.shift + sample * a.shift_stride + c, sh);
    if (a.weight_after && there) eight_of(a.weight_after, c, wa);
    if (a.weight && there) eight_of(a.weight, c, wb);
    f32x2 p[4], q[4], f[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) p[k] = f2u(g[2 * k], g[2 * k + 1]), q[k] = f2u(1.f + sc[2 * k], 1.f + sc[2 * k + 1]);
    if (a.weight_after && there) {
      wa.get(f);
#pragma unroll
      for (int k = 0; k < 4; ++k) p[k] = fmul2(p[k], f[k]);
    }
    if (a.weight && there) {
      wb.get(f);
#pragma unroll
      for (int k = 0; k < 4; ++k) q[k] = fmul2(q[k], f[k]);
    }
    const int at = (c & ~255) + (c & 248) / 2;   // the first four; the others 128 places behind
    auto put = [&](float* to, f32x2 v0, f32x2 v1, f32x2 v2, f32x2 v3) {
      *reinterpret_cast<ulonglong2*>(to + at) = make_ulonglong2(v0, v1);
      *reinterpret_cast<ulonglong2*>(to + at + 128) = make_ulonglong2(v2, v3);
    };
    put(fp, p[0], p[1], p[2], p[3]);
    put(fq, q[0], q[1], q[2], q[3]);
    if (has_s) put(fs, f2u(sh[0], sh[1]), f2u(sh[2], sh[3]), f2u(sh[4], sh[5]), f2u(sh[6], sh[7]));
  }
  if (threadIdx.x < 64) sums[0][0][threadIdx.x] = sums[0][1][threadIdx.x] = sums[1][0][threadIdx.x] = sums[1][1][threadIdx.x] = 0.f;
  __syncthreads();
  auto factor = [&](const float* f, int i, f32x2 (&v)[4]) {
    const ulonglong2* p = reinterpret_cast<const ulonglong2*>(f + (w * NB + i) * 256 + 4 * lane);
    const ulonglong2 l = p[0], h = p[32];
    v[0] = l.x, v[1] = l.y, v[2] = h.x, v[3] = h.y;
  };

  // Mean (0 where the norm has none) and 1 / root mean square of a row's columns, the which-th norm of the
  // row; a warp finds its own mean and squares around it first.  A warp that writes one norm's sums has passed the
  // other's barrier, behind which all have read the row before's.
  auto held = [&](int k) { return (float)max(0, min(C, (k + 1) * NB * 256) - k * NB * 256); };   // columns of a warp
  const float per_col = 1.f / (float)C, mine = held(w), per_mine = mine > 0.f ? 1.f / mine : 0.f;
  auto norm = [&](const f32x2 (&v)[NB][4], int which) {
    float mean = 0.f, ss;
    f32x2 sum = 0, more = 0;
    if (a.centered) {
#pragma unroll
      for (int i = 0; i < NB; ++i) sum = fadd2(sum, fadd2(fadd2(v[i][0], v[i][1]), fadd2(v[i][2], v[i][3])));
      mean = warp_sum(lo_f(sum) + hi_f(sum)) * per_mine;
      const f32x2 m2 = f2u(-mean, -mean);
      sum = 0;
#pragma unroll
      for (int i = 0; i < NB; ++i)
        if (in[i])
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const f32x2 d = fadd2(v[i][k], m2);
            sum = ffma2(d, d, sum);
          }
    } else {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        sum = ffma2(v[i][1], v[i][1], ffma2(v[i][0], v[i][0], sum));
        more = ffma2(v[i][3], v[i][3], ffma2(v[i][2], v[i][2], more));
      }
      sum = fadd2(sum, more);
    }
    ss = warp_sum(lo_f(sum) + hi_f(sum));
    if (W > 1) {
      float *of = &sums[which][0][8 * slot], *means = &sums[which][1][8 * slot];
      if (lane == 0) {
        of[w] = ss;
        if (a.centered) means[w] = mean;
      }
      slot_sync(slot, W);
      const float4 s0 = reinterpret_cast<const float4*>(of)[0], s1 = reinterpret_cast<const float4*>(of)[1];
      ss = ((s0.x + s0.y) + (s0.z + s0.w)) + ((s1.x + s1.y) + (s1.z + s1.w));
      if (a.centered) {
        float m = 0.f;
        for (int k = 0; k < W; ++k) m = fmaf(means[k], held(k), m);
        mean = m * per_col;
        for (int k = 0; k < W; ++k) ss = fmaf((means[k] - mean) * (means[k] - mean), held(k), ss);
      }
    }
    return make_float2(mean, rsqrtf(fmaf(ss, per_col, a.eps)));
  };
  // The row without its mean, where it has one, and 1 / root mean square for both of a pair.
  auto normed = [&](f32x2 (&v)[NB][4], float2 n) {
    if (a.centered) {
      const f32x2 m2 = f2u(-n.x, -n.x);
#pragma unroll
      for (int i = 0; i < NB; ++i)
        if (in[i])
#pragma unroll
          for (int k = 0; k < 4; ++k) v[i][k] = fadd2(v[i][k], m2);
    }
    return f2u(n.y, n.y);
  };

  const f32x2 rs = f2u(a.resid_scale, a.resid_scale);
  T* sm = reinterpret_cast<T*>(a.sum) + (first + slot) * a.ldsum + c0;
  T* o = reinterpret_cast<T*>(a.out) + (first + slot) * a.ldo + c0;
  uint8_t* o8 = reinterpret_cast<uint8_t*>(a.q8.q) + (first + slot) * a.q8.ldq + c0;
  float* sp = a.q8.scale + (long long)(w * NB * 2 + (lane >> 4)) * a.q8.lds + first + slot;
  const bool alone = W > 1 && !(a.norm_after && (Q8 || a.out));   // one norm to a row: it has no other's barrier
  for (long long r = first + slot; r < end; r += slots) {
    if (alone) slot_sync(slot, W);
    f32x2 h[NB][4], res[NB][4];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      fy[i].get(h[i]);
      fx[i].get(res[i]);
    }
    if (r + slots < end) load_row();
    f32x2 by = f2u(1.f, 1.f);
    if (a.norm_after) by = normed(h, norm(h, 0));
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      f32x2 p[4];
      factor(fp, i, p);
#pragma unroll
      for (int k = 0; k < 4; ++k) h[i][k] = ffma2(rs, res[i][k], fmul2(h[i][k], fmul2(by, p[k])));
      if (ragged && !in[i]) h[i][0] = h[i][1] = h[i][2] = h[i][3] = 0;
      if (a.sum && in[i]) Cols<T>::store(sm + 256 * i, h[i]);
    }
    sm += a.ldsum * slots;
    if (!Q8 && !a.out) continue;
    by = normed(h, norm(h, 1));
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      f32x2 q[4], s[4];
      factor(fq, i, q);
      if (has_s) {
        factor(fs, i, s);
#pragma unroll
        for (int k = 0; k < 4; ++k) h[i][k] = ffma2(h[i][k], fmul2(by, q[k]), s[k]);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) h[i][k] = fmul2(h[i][k], fmul2(by, q[k]));
      }
    }
    if constexpr (!Q8) {
#pragma unroll
      for (int i = 0; i < NB; ++i)
        if (in[i]) Cols<T>::store(o + 256 * i, h[i]);
      o += a.ldo * slots;
    } else {
#pragma unroll
      for (int i = 0; i < NB; ++i) {   // 16 lanes to a scale
        float m = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) m = max_abs(m, max_abs(lo_f(h[i][k]), hi_f(h[i][k])));
        if (!in[i]) m = 0.f;
#pragma unroll
        for (int k = 8; k; k >>= 1) m = max_abs(m, __shfl_xor_sync(0xffffffffu, m, k));
        const float sc = q8_scale(__float_as_uint(m)), inv = q8_inv(sc);
        if (in[i]) {
          const f32x2 i2 = f2u(inv, inv);
          f32x2 v[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = fmul2(h[i][k], i2);
          *reinterpret_cast<uint2*>(o8 + 256 * i) = make_uint2(to_e4m3x4(lo_f(v[0]), hi_f(v[0]), lo_f(v[1]), hi_f(v[1])),
                                                                to_e4m3x4(lo_f(v[2]), hi_f(v[2]), lo_f(v[3]), hi_f(v[3])));
          if ((lane & 15) == 0) sp[2 * i * a.q8.lds] = sc;
        }
      }
      o8 += a.q8.ldq * slots;
      sp += slots;
    }
  }
}

// Rows on any boundary and of any width, element by element: NB adjacent 128-column blocks to a warp,
// adjacent rows one after the other.  With KEEP the factors stay in registers until the sample changes.
// Bound by the latency of single elements' loads and of the norms' meetings: 1333 x 1001 in fp32, centered
// and modulated, 8.4 us, 2.5 TB/s; 14566 x 1001 in bf16 55 us.
template <class T, int NB, bool Q8, bool KEEP>
__global__ void __launch_bounds__(256, KEEP ? 2 : 1) k_block_norms_any(long long rows, int C, int W, long long per,
                                                                   const __grid_constant__ BlockNormsArgs a) {
  __shared__ float2 red[2][8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, w = warp & (W - 1), slot = warp / W;
  const int c0 = w * NB * 128 + lane, left = C - c0;   // columns from the lane's first on
  const int held = min(C, (w + 1) * NB * 128) - w * NB * 128;   // columns of the warp; none where not positive
  const long long r0 = ((long long)blockIdx.x * (8 / W) + slot) * per, r1 = min(rows, r0 + per);
  Four<T, false> fy[NB], fx[NB];
  f32x2 p[KEEP ? NB : 1][2], q[KEEP ? NB : 1][2], s[KEEP ? NB : 1][2];
  long long sample = -1;
  pdl_trigger();
  pdl_wait();
  const T* y = reinterpret_cast<const T*>(a.y) + r0 * a.ldy + c0;   // of the next row to load
  const T* x = reinterpret_cast<const T*>(a.x) + r0 * a.ldx + c0;
  auto load_row = [&] {
#pragma unroll
    for (int i = 0; i < NB; ++i)
      if (128 * i < left) {
        fy[i].load(y + 128 * i, left - 128 * i);
        if (a.x) fx[i].load(x + 128 * i, left - 128 * i);
      }
    y += a.ldy;
    x += a.ldx;
  };
  // the three factors of a lane's four columns of block i, for this row's sample
  auto times = [&](f32x2 (&v)[2], const void* weight, int i) {
    if (!weight) return;
    Four<T, false> f;
    f32x2 u[2];
    f.load(reinterpret_cast<const T*>(weight) + c0 + 128 * i, left - 128 * i);
    f.get(u);
    v[0] = fmul2(v[0], u[0]);
    v[1] = fmul2(v[1], u[1]);
  };
  auto four = [&](const float* m, long long stride, int i, f32x2 (&v)[2]) {   // (of fp32 rows, on any boundary)
    m += sample * stride + c0 + 128 * i;
    float e[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) e[k] = 32 * k < left - 128 * i ? m[32 * k] : 0.f;
    v[0] = f2u(e[0], e[1]);
    v[1] = f2u(e[2], e[3]);
  };
  const f32x2 one = f2u(1.f, 1.f);
  auto make_p = [&](int i, f32x2 (&v)[2]) {
    v[0] = v[1] = one;
    if (128 * i >= left) return;
    if (a.gate) four(a.gate, a.gate_stride, i, v);
    times(v, a.weight_after, i);
  };
  auto make_qs = [&](int i, f32x2 (&v)[2], f32x2 (&u)[2]) {
    v[0] = v[1] = one;
    u[0] = u[1] = 0;
    if (128 * i >= left) return;
    if (a.scale) {
      four(a.scale, a.scale_stride, i, v);
      v[0] = fadd2(v[0], one);
      v[1] = fadd2(v[1], one);
    }
    if (a.shift) four(a.shift, a.shift_stride, i, u);
    times(v, a.weight, i);
  };
  // a pair of columns, 0 past the row's end
  auto within = [&](f32x2 v, int i, int k) -> f32x2 {
    return 128 * i + 64 * k + 32 < left ? v : 128 * i + 64 * k < left ? f2u(lo_f(v), 0.f) : 0;
  };
  // mean (0 where the norm has none) and 1 / root mean square of a row's columns; a warp finds its own mean and
  // squares around it first; two places take turns, so that a warp that writes one has passed the barrier behind
  // which all others had read it
  int turn = 0;
  auto norm = [&](const f32x2 (&v)[NB][2]) {
    float mean = 0.f, ss;
    f32x2 sum = 0;
    if (a.centered) {
#pragma unroll
      for (int i = 0; i < NB; ++i) sum = fadd2(sum, fadd2(v[i][0], v[i][1]));
      mean = held > 0 ? warp_sum(lo_f(sum) + hi_f(sum)) / (float)held : 0.f;
      const f32x2 m2 = f2u(-mean, -mean);
      sum = 0;
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const f32x2 d = within(fadd2(v[i][k], m2), i, k);
          sum = ffma2(d, d, sum);
        }
    } else {
#pragma unroll
      for (int i = 0; i < NB; ++i) sum = ffma2(v[i][1], v[i][1], ffma2(v[i][0], v[i][0], sum));
    }
    ss = warp_sum(lo_f(sum) + hi_f(sum));
    if (W > 1) {
      float2* of = red[turn];
      turn ^= 1;
      if (lane == 0) of[warp] = make_float2(mean, ss);
      slot_sync(slot, W);
      float all = 0.f, m = 0.f;
      if (a.centered) {
        for (int k = 0; k < W; ++k) m += of[warp - w + k].x * (float)max(0, min(C, (k + 1) * NB * 128) - k * NB * 128);
        m /= (float)C;
      }
      for (int k = 0; k < W; ++k) {
        const float2 o = of[warp - w + k];
        all += o.y;
        if (a.centered) all = fmaf((o.x - m) * (o.x - m), (float)max(0, min(C, (k + 1) * NB * 128) - k * NB * 128), all);
      }
      mean = m;
      ss = all;
    }
    return make_float2(mean, rsqrtf(ss / (float)C + a.eps));
  };

  // The row without its mean, where it has one, and 1 / root mean square for both of a pair.
  auto normed = [&](f32x2 (&v)[NB][2], float2 n) {
    if (a.centered) {
      const f32x2 m2 = f2u(-n.x, -n.x);
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int k = 0; k < 2; ++k) v[i][k] = within(fadd2(v[i][k], m2), i, k);
    }
    return f2u(n.y, n.y);
  };
  const f32x2 rs = f2u(a.resid_scale, a.resid_scale);

  if (r0 < r1) load_row();
  long long to = 0;   // rows of the sample end here
  T* sm = reinterpret_cast<T*>(a.sum) + r0 * a.ldsum + c0;
  T* o = reinterpret_cast<T*>(a.out) + r0 * a.ldo + c0;
  uint8_t* o8 = reinterpret_cast<uint8_t*>(a.q8.q) + r0 * a.q8.ldq + c0;
  float* sp = a.q8.scale + (long long)(w * NB) * a.q8.lds + r0;
  for (long long r = r0; r < r1; ++r) {
    if (r >= to) {
      sample = (a.gate || a.scale || a.shift) ? r / a.rpb : 0;
      to = (a.gate || a.scale || a.shift) ? (sample + 1) * a.rpb : rows;
      if constexpr (KEEP) {
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          make_p(i, p[i]);
          make_qs(i, q[i], s[i]);
        }
      }
    }
    f32x2 h[NB][2], res[NB][2];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      h[i][0] = h[i][1] = res[i][0] = res[i][1] = 0;
      if (128 * i < left) {
        fy[i].get(h[i]);
        if (a.x) fx[i].get(res[i]);
      }
    }
    if (KEEP && r + 1 < r1) load_row();
    f32x2 by = one;
    if (a.norm_after) by = normed(h, norm(h));
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      if constexpr (!KEEP) make_p(i, p[0]);
#pragma unroll
      for (int k = 0; k < 2; ++k) h[i][k] = ffma2(rs, res[i][k], fmul2(h[i][k], fmul2(by, p[KEEP ? i : 0][k])));
      if (a.sum && 128 * i < left) Four<T, false>::store(sm + 128 * i, left - 128 * i, h[i]);
    }
    sm += a.ldsum;
    if (!Q8 && !a.out) continue;
    by = normed(h, norm(h));
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      if constexpr (!KEEP) make_qs(i, q[0], s[0]);
#pragma unroll
      for (int k = 0; k < 2; ++k) h[i][k] = ffma2(h[i][k], fmul2(by, q[KEEP ? i : 0][k]), s[KEEP ? i : 0][k]);
    }
    if constexpr (!Q8) {
#pragma unroll
      for (int i = 0; i < NB; ++i)
        if (128 * i < left) Four<T, false>::store(o + 128 * i, left - 128 * i, h[i]);
      o += a.ldo;
    } else {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        // columns past the row's end hold no magnitude
        float m = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (128 * i + 32 * k < left) m = max_abs(m, k & 1 ? hi_f(h[i][k / 2]) : lo_f(h[i][k / 2]));
        const float sc = q8_scale(__reduce_max_sync(0xffffffffu, __float_as_uint(m)));
        if (128 * i < left) ff::store8<false>(o8 + 128 * i, left - 128 * i, h[i], q8_inv(sc));
        if (lane == 0 && 128 * i < held) sp[i * a.q8.lds] = sc;
      }
      o8 += a.q8.ldq;
      ++sp;
    }
  }
}

// pieces (256 columns, or 128 element by element) to a warp of the rows' eight at most
constexpr int PIECES_MAX = BLOCK_NORMS_COLS_MAX / 256 / 8, ANY_MAX = BLOCK_NORMS_COLS_MAX / 128 / 8;

template <class T, int NB, bool Q8> cudaError_t norms_any_nb(int W, long long rows, int C, const BlockNormsArgs& a, cudaStream_t s) {
  constexpr bool KEEP = NB <= 2;
  const int slots = 8 / W;
  // two blocks to an SM go over all rows where factors stay in registers; else a row to a slot
  const long long most = KEEP ? 152 * 2 : (rows + slots - 1) / slots, per = (rows + most * slots - 1) / (most * slots);
  const long long grid = (rows + per * slots - 1) / (per * slots);
  const cudaError_t e = launch_pdl(k_block_norms_any<T, NB, Q8, KEEP>, (unsigned)grid, 256, 0, s, rows, C, W, per, a);
  return e != cudaSuccess ? e : launched();
}
template <class T, bool Q8> cudaError_t norms_any(long long rows, int C, const BlockNormsArgs& a, cudaStream_t s) {
  const int blocks = (C + 127) / 128;
  // two blocks to a warp, fewer while the rows alone leave the SMs without 8 warps each
  int W = 1;
  while (W < 8 && (blocks > 2 * W || (rows * W < 152 * 8 && blocks > W))) W *= 2;
  const int nb = (blocks + W - 1) / W;
  return nb <= 1 ? norms_any_nb<T, 1, Q8>(W, rows, C, a, s) : nb <= 2 ? norms_any_nb<T, 2, Q8>(W, rows, C, a, s)
         : nb <= 4 ? norms_any_nb<T, 4, Q8>(W, rows, C, a, s) : norms_any_nb<T, ANY_MAX, Q8>(W, rows, C, a, s);
}

template <class T, int NB, bool Q8> cudaError_t norms_nb(int W, long long rows, int C, BlockNormsArgs a, cudaStream_t s) {
  const auto kernel = k_block_norms<T, NB, Q8>;
  const int wide = W * NB * 256, slots = 8 / W;
  const bool modulated = a.gate || a.scale || a.shift;
  if (!modulated) a.rpb = (int)rows;
  const size_t smem = 4ull * wide * (2 + (a.shift != nullptr));
  // (the limit of the widest row, set once: another call of the process may come between it and a launch)
  static PerDevice<int> limits;
  int dev = 0, limit = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= PerDevice<int>::devices) return cudaErrorNotSupported;
  e = limits.get(dev, &limit, [&](int& v) {
    v = 12 * std::min(NB * 2048, BLOCK_NORMS_COLS_MAX);
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, v);
  });
  if (e != cudaSuccess) return e;
  // rows of a sample in chunks: as many blocks as the SMs hold at once, or a row to a slot
  const long long samples = (rows + a.rpb - 1) / a.rpb, held = 152ll * NORMS_BLOCKS<T, NB>;
  const long long of_sample = std::min<long long>(rows, a.rpb), want = std::max(1ll, held / samples);
  const long long per = std::max<long long>(slots, ((of_sample + want - 1) / want + slots - 1) / slots * slots);
  const long long chunks = (of_sample + per - 1) / per;
  if (samples * chunks > 0x7fffffff) return cudaErrorInvalidValue;
  e = launch_pdl(kernel, (unsigned)(samples * chunks), 256, smem, s, rows, C, W, per, (int)chunks, a);
  return e != cudaSuccess ? e : launched();
}
template <class T, bool Q8> cudaError_t norms(long long rows, int C, const BlockNormsArgs& a, cudaStream_t s) {
  const auto al = [](const void* p, long long ld) { return !((uintptr_t)p & 15) && ld % (16 / (int)sizeof(T)) == 0; };
  // (few rows with weights alone too: 1, 152 and 304 rows of 2048 in bf16 with 8-bit output 2.4, 2.6 and 2.9 us, element
  // by element 3.0, 3.5 and 3.7; of 512 columns 2.15, 2.42 and 2.40, and 2.04, 2.40 and 2.64)
  if (C % 8 || !al(a.y, a.ldy) || (a.x && !al(a.x, a.ldx)) || (a.sum && !al(a.sum, a.ldsum)) || (a.out && !al(a.out, a.ldo)))
    return norms_any<T, Q8>(rows, C, a, s);
  const int pieces = (C + 255) / 256;
  // Warps to a row: four pieces to a warp, fewer while the rows alone leave the SMs without 8 warps each.
  // 14566 x 2048 with modulation and 8-bit output 35.8 us with four, 38.9 with eight (one block to an SM), before the
  // factors' present form 38.0 and 45.8 with two; fp32 85.3, with two 84.5, centered 79.5 and 86.5.
  constexpr int PREF = 4;
  int W = 1;
  while (W < 8 && (pieces > PREF * W || (rows * W < 152 * 8 && pieces > W))) W *= 2;
  const int nb = (pieces + W - 1) / W;
  return nb <= 1 ? norms_nb<T, 1, Q8>(W, rows, C, a, s) : nb <= 2 ? norms_nb<T, 2, Q8>(W, rows, C, a, s)
         : nb <= 3 ? norms_nb<T, 3, Q8>(W, rows, C, a, s) : nb <= 4 ? norms_nb<T, 4, Q8>(W, rows, C, a, s)
                   : norms_nb<T, PIECES_MAX, Q8>(W, rows, C, a, s);
}

}  // namespace

cudaError_t launch_block_norms(DType dt, long long rows, int C, const BlockNormsArgs& a, cudaStream_t s) {
  const bool q8 = a.q8.q != nullptr;
  return dt == F32 ? (q8 ? norms<float, true>(rows, C, a, s) : norms<float, false>(rows, C, a, s))
                   : (q8 ? norms<bf16, true>(rows, C, a, s) : norms<bf16, false>(rows, C, a, s));
}

}  // namespace ff
