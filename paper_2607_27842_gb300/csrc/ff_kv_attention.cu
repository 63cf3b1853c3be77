// Attention of one new token of each sequence over the 8-bit key-value cache
// (formulas: featfix_op_kv_attention).  Bound by memory: every cached byte that a token
// sees is read once for all query heads of its key head.
//
// The work is a line of steps: a unit is one key head of one sequence with up to 8 or 16 of
// its query heads, a step T of its tokens; the units of a sequence follow one another, then
// the next sequence's.  Every warp of the grid takes an equal stretch of the line,
// whatever the lengths are, and goes over it on its own: tokens come by asynchronous
// copies, one or more steps ahead, to a place that only the copying lane reads (so
// shared memory has no layout to agree on and no bank conflicts); e4m3 becomes fp16 in
// registers, exactly; products are mma.sync m16n8k16 with tokens or columns as the 16 and
// query heads as the 8, because a token's few query heads would fill 4 of tcgen05's 128
// rows, and the products are far from a bound here.
//
//   S^T[token, query] = K Q^T,   O^T[column, query] += V^T P^T
//
// Sums over any index may go in any order as long as both factors agree on it: lane (g, j) =
// (lane / 4, lane % 4) holds 16 adjacent columns of keys g and g + 8, and for the second
// product 16 adjacent columns of values 2j, 2j + 1, 2j + 8, 2j + 9, whole 16-byte vectors in the
// order of memory.  P^T turns from the one's result to the other's operand in movmatrix.
//
// Softmax with a running maximum m of the scores x (in powers of two).  The weights p * scale_v
// go to fp16, times 2^(m + 15 - mw) with a running maximum mw of x + log2(scale_v): the largest
// weight uses all of fp16's range whatever the scales are, and weights 2^-29 below it still
// have 11 bits.  The softmax's sum takes p = exp2(x - m) in fp32.
//
// A stretch begins and ends within units.  What belongs to one unit of several warps meets in
// shared memory at the end, and of several blocks in the workspace, which a second
// kernel adds in the line's order: no atomics, the same bits every time.
#include "ff_kv8.cuh"
#include "ff_host.h"

#include <cuda_fp16.h>

#include <algorithm>

namespace ff {

namespace {

constexpr int WARPS = 8;
constexpr int GRID_MAX = 160;      // blocks that the workspace has room for
constexpr float NONE = -3.0e38f;   // maximum of nothing
// longest units, in steps, of which every block takes whole ones (no second kernel)
constexpr int WHOLE_STEPS = 32;

// Shapes of a variant: columns of a head rounded up to DP, NT times 8 query heads.
template <int DP, int NT> struct Shape {
  static constexpr int MT = DP == 256 ? 1 : 2;                 // groups of 16 tokens in a step
  static constexpr int T = 16 * MT;
  static constexpr int STAGES = DP == 64 ? 4 : 2;
  static constexpr int NK = DP / 64;                           // 16-byte vectors of a key to a lane
  static constexpr int VB = DP >= 128 ? 16 : 8;                // bytes of a value's vector
  static constexpr int NV = DP / 8 / VB;
  static constexpr int STAGE = T * DP * 2 + T * 8 + 16;        // keys, values, scales, mask
  static constexpr int RING = STAGE * STAGES;                  // of a warp
  static constexpr int NQ = 8 * NT;
  static constexpr int PART = NQ * (DP + 4);                   // floats: sums, then m, l, mw of each query
  static constexpr int SMEM = WARPS * (RING + PART * 4);
  static_assert(PART * 4 <= RING, "the second partial result lies in the ring");
  static_assert(STAGE % 16 == 0 && PART % 4 == 0, "whole vectors");
};

struct Plan {
  unsigned div_m, div_s;   // token / page_size
  int group, tiles;        // query heads of a key head, units that share them
  int whole;               // blocks take whole units
  int pairs;               // results may be stored in pairs
  float scale;             // softmax scale times log2(e)
};

__device__ __forceinline__ unsigned cvt_e4m3x2(unsigned short u) {
  unsigned r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(u));
  return r;
}
__device__ __forceinline__ void mma16816(float (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ unsigned transposed8x8(unsigned x) {
  unsigned r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float lg2(float x) {
  float r;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ unsigned half2_bits(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const unsigned*>(&h);
}
__device__ __forceinline__ void cp_async8(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async16s(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async4s(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// Tokens that sequence b's new token sees.
struct Seen {
  int first, end;
};
__device__ __forceinline__ Seen seen(const KvCache& c, int window, int b) {
  const int len = kv_len(c, b);
  return {window && len > window ? len - window : 0, len};
}

// Where a step of the line is: sequence, unit of it, step of the unit, steps of the unit.
struct Spot {
  int b, unit;
  int step, steps;
};

// Steps of all sequences before those of each thread's share (exclusive sums in shared
// memory, the line's length behind them).
__device__ __forceinline__ int share(int seqs) { return (seqs + 32 * WARPS - 1) / (32 * WARPS); }
template <int T> __device__ void line_up(const KvCache& c, int window, int units, long long* before, long long* warp_sum) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, per = share(c.seqs);
  long long n = 0;
  for (int i = 0; i < per; ++i) {
    const int b = tid * per + i;
    if (b < c.seqs) {
      const Seen s = seen(c, window, b);
      n += (s.end - s.first + T - 1) / T;
    }
  }
  n *= units;
  long long sum = n;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += v;
  }
  if (lane == 31) warp_sum[warp] = sum;
  __syncthreads();
  long long base = 0;
  for (int w = 0; w < warp; ++w) base += warp_sum[w];
  before[tid] = base + sum - n;
  if (tid == 32 * WARPS - 1) before[32 * WARPS] = base + sum;
  __syncthreads();
}
// The spot of step `at` of the line (below its length).
template <int T>
__device__ Spot locate(const KvCache& c, int window, int units, const long long* before, long long at) {
  int lo = 0, hi = 32 * WARPS;   // the last share that starts at or before `at`
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (before[mid] <= at) lo = mid;
    else hi = mid;
  }
  at -= before[lo];
  for (int b = lo * share(c.seqs); b < c.seqs; ++b) {
    const Seen s = seen(c, window, b);
    const int steps = (s.end - s.first + T - 1) / T;
    if (at < (long long)steps * units) {
      const int unit = (int)(at / steps);
      return {b, unit, (int)(at - (long long)unit * steps), steps};
    }
    at -= (long long)steps * units;
  }
  return {c.seqs - 1, 0, 0, 1};   // (lengths that change meanwhile: no address out of range)
}

// The unit behind the one at s that has steps.
template <int T> __device__ __forceinline__ void next_unit(const KvCache& c, int window, int units, Spot& s) {
  s.step = 0;
  if (++s.unit < units) return;
  s.unit = 0;
  do {
    if (s.b + 1 >= c.seqs) return;   // (as above: the line has an end before)
    const Seen e = seen(c, window, ++s.b);
    s.steps = (e.end - e.first + T - 1) / T;
  } while (s.steps == 0);
}

// Two columns of a result, in one store where addresses allow it.
template <class T>
__device__ __forceinline__ void store_row(T* out, int pairs, int col, int dim, float x, float y) {
  if (pairs) {
    if (col >= dim) return;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<__nv_bfloat162*>(out + col) = __floats2bfloat162_rn(x, y);
    else *reinterpret_cast<float2*>(out + col) = make_float2(x, y);
  } else {
    if (col < dim) out[col] = from_f<T>(x);
    if (col + 1 < dim) out[col + 1] = from_f<T>(y);
  }
}
// 2^(mw - m - 15) / l, by which sums become results; 0 for a row of no tokens
__device__ __forceinline__ float closing(float m, float l, float mw) {
  return l == 0.f ? 0.f : ex2(mw - m - 15.f) / l;
}
__device__ __forceinline__ float lse_of(float m, float l) {
  return l == 0.f ? __int_as_float(0xff800000) : (m + log2f(l)) * 0.69314718055994531f;
}

template <class T, int DP, int NT>
__global__ void __launch_bounds__(32 * WARPS, 1) k_kv_attention(const __grid_constant__ KvCache c,
                                                                 const __grid_constant__ KvAttnArgs a,
                                                                 const __grid_constant__ Plan p) {
  typedef Shape<DP, NT> Sh;
  constexpr int TERMS = sizeof(T) == 4 ? 2 : 1;   // fp16 terms of queries and of weights
  extern __shared__ __align__(16) char smem[];
  __shared__ long long before[32 * WARPS + 1], warp_sum[WARPS];
  __shared__ int part_unit[WARPS][2][2];          // sequence and unit of a warp's partial results, -1: none
  __shared__ int part_ends[WARPS];                // whether the first of them has its unit's last step
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, j = lane & 3;
  const int units = c.heads * p.tiles, dim = c.head_dim;
  pdl_trigger();
  pdl_wait();

  // rows of sequences without tokens
  for (int b = blockIdx.x; b < c.seqs; b += gridDim.x) {
    const Seen s = seen(c, a.window, b);
    if (s.end > s.first) continue;
    T* out = reinterpret_cast<T*>(a.out) + b * a.ldo;
    for (int i = threadIdx.x; i < a.q_heads * dim; i += 32 * WARPS) out[i] = from_f<T>(0.f);
    if (a.lse)
      for (int i = threadIdx.x; i < a.q_heads; i += 32 * WARPS) a.lse[(long long)b * a.q_heads + i] = __int_as_float(0xff800000);
  }

  line_up<Sh::T>(c, a.window, units, before, warp_sum);
  const long long total = before[32 * WARPS];
  // blocks that have a share: with a step to every warp
  const long long blocks = max(1ll, min((long long)gridDim.x, (total + WARPS - 1) / WARPS));
  auto edge = [&](long long i) {   // of block i: its first step of the line
    long long at = total * min(i, blocks) / blocks;
    if (p.whole && at < total) {
      const Spot s = locate<Sh::T>(c, a.window, units, before, at);
      if (s.step) at += s.steps - s.step;
    }
    return at;
  };
  const long long c0 = edge(blockIdx.x), c1 = edge(blockIdx.x + 1ll);
  // (rounded up: the first warp has steps where any has)
  const long long w0 = c0 + ((c1 - c0) * warp + WARPS - 1) / WARPS, w1 = c0 + ((c1 - c0) * (warp + 1) + WARPS - 1) / WARPS;
  if (lane == 0) part_unit[warp][0][0] = part_unit[warp][1][0] = -1, part_ends[warp] = 0;

  char* ring = smem + warp * Sh::RING;
  float* part0 = reinterpret_cast<float*>(smem + WARPS * Sh::RING) + warp * Sh::PART;
  float* part1 = reinterpret_cast<float*>(ring);
  const uint32_t ring_s = (uint32_t)__cvta_generic_to_shared(ring);

  if (w0 < w1) {
    Spot in = locate<Sh::T>(c, a.window, units, before, w0), at = in;
    int to_issue = (int)min((long long)0x7fffffff, w1 - w0), to_do = to_issue;
    Seen in_seen = seen(c, a.window, in.b);

    // Page of this lane's token of the step at `in`, looked up one step before its copies.
    auto token = [&] { return in_seen.first + in.step * Sh::T + (lane & (Sh::T - 1)); };
    auto page_of = [&](int t) { return (int)((__umulhi(p.div_m, (unsigned)t) + (unsigned)t) >> p.div_s); };
    auto look_up = [&] {
      const int t = token();
      return t < in_seen.end ? c.table[in.b * c.ld_table + page_of(t)] : -1;
    };
    int entry = look_up();
    int stage_in = 0;
    auto issue = [&] {
      if (to_issue > 0) {
        const int t = token(), slot = t - page_of(t) * c.page_size;
        const bool there = (unsigned)entry < (unsigned)c.pages && t < in_seen.end;
        const long long page = there ? entry : 0, sl = there ? slot : 0;
        const unsigned mask = __ballot_sync(0xffffffffu, there);
        const int head = in.unit / p.tiles;
        const long long ko = page * c.k_stride[0] + sl * c.k_stride[1], vo = page * c.v_stride[0] + sl * c.v_stride[1];
        const char* kb = reinterpret_cast<const char*>(c.k) + head * c.k_stride[2];
        const char* vb = reinterpret_cast<const char*>(c.v) + head * c.v_stride[2];
        const uint32_t st = ring_s + stage_in * Sh::STAGE;
#pragma unroll
        for (int mt = 0; mt < Sh::MT; ++mt)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int k = 16 * mt + 8 * r + g;
            const char* src = kb + __shfl_sync(0xffffffffu, ko, k);
            const bool ok = mask >> k & 1;
#pragma unroll
            for (int i = 0; i < Sh::NK; ++i) {
              const int col = 16 * (j + 4 * i), n = ok ? min(16, max(0, dim - col)) : 0;
              cp_async16s(st + ((mt * 2 + r) * Sh::NK + i) * 512 + lane * 16, src + (n ? col : 0), n);
            }
          }
        const uint32_t sv = st + Sh::T * DP;
#pragma unroll
        for (int mt = 0; mt < Sh::MT; ++mt)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int k = 16 * mt + 8 * (r >> 1) + 2 * j + (r & 1);
            const char* src = vb + __shfl_sync(0xffffffffu, vo, k);
            const bool ok = mask >> k & 1;
#pragma unroll
            for (int i = 0; i < Sh::NV; ++i) {
              const int col = DP / 8 * g + Sh::VB * i, n = ok ? min(Sh::VB, max(0, dim - col)) : 0;
              const uint32_t dst = sv + ((mt * 4 + r) * Sh::NV + i) * (32 * Sh::VB) + lane * Sh::VB;
              if constexpr (Sh::VB == 16) cp_async16s(dst, src + (n ? col : 0), n);
              else cp_async8(dst, src + (n ? col : 0), n);
            }
          }
        const uint32_t ss = st + Sh::T * DP * 2;
        if (lane < Sh::T) {
          cp_async4s(ss + 4 * lane, c.k_scale + (page * c.k_scale_stride[0] + sl * c.k_scale_stride[1] + head * c.k_scale_stride[2]),
                     there ? 4 : 0);
          cp_async4s(ss + 4 * (Sh::T + lane),
                     c.v_scale + (page * c.v_scale_stride[0] + sl * c.v_scale_stride[1] + head * c.v_scale_stride[2]), there ? 4 : 0);
        }
        if (lane == 0) *reinterpret_cast<unsigned*>(ring + stage_in * Sh::STAGE + Sh::T * DP * 2 + Sh::T * 8) = mask;
        stage_in = stage_in + 1 == Sh::STAGES ? 0 : stage_in + 1;
        if (--to_issue > 0) {
          if (++in.step == in.steps) {
            next_unit<Sh::T>(c, a.window, units, in);
            in_seen = seen(c, a.window, in.b);
          }
          entry = look_up();
        }
      }
      cp_commit();   // (an empty group keeps the count)
    };
#pragma unroll
    for (int i = 0; i < Sh::STAGES; ++i) issue();

    unsigned qf[NT][TERMS][DP / 16][2];
    float qs[NT][2];                         // of queries 2j, 2j + 1: what a product is multiplied by
    float m[NT][2], l[NT][2], mw[NT][2], o[NT][DP / 16][4];
    int stage = 0, begun = at.step == 0;     // whether this warp has the unit's first step
    bool fresh = true;
    while (to_do > 0) {
      if (fresh) {
        fresh = false;
        const int head = at.unit / p.tiles, tile = at.unit - head * p.tiles;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          // query g of the tile: four adjacent columns for each 16 of the sum
          const int qi = tile * Sh::NQ + nt * 8 + g;
          const T* q = reinterpret_cast<const T*>(a.q) + at.b * a.ldq + (long long)(head * p.group + qi) * dim;
          float x[DP / 16][4], top = 0.f;
#pragma unroll
          for (int s = 0; s < DP / 16; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int col = 16 * (j + 4 * (s / 4)) + 4 * (s % 4) + e;
              x[s][e] = qi < p.group && col < dim ? to_f(q[col]) : 0.f;
              top = max_abs(top, x[s][e]);
            }
          top = max_abs(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = max_abs(top, __shfl_xor_sync(0xffffffffu, top, 2));
          // a power of two brings the largest to 2^14 .. 2^15: the terms below lose nothing above
          // 2^-40 (in two terms 2^-23) of it.  Infinities and NaN become NaN.
          const int ex = max(-100, min(127, (int)(__float_as_uint(top) >> 23 & 0xff) - 127));
          float up = __int_as_float((max(-126, 14 - ex) + 127) << 23), down = __int_as_float((max(-126, ex - 14) + 127) << 23);
          if (!(top < __int_as_float(0x7f800000))) up = __int_as_float(0x7fffffff);
          if (ex == -100 && top == 0.f) up = down = 1.f;
#pragma unroll
          for (int s = 0; s < DP / 16; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float u = x[s][2 * h] * up, v = x[s][2 * h + 1] * up;
              qf[nt][0][s][h] = half2_bits(u, v);
              if constexpr (TERMS == 2) {
                const float2 hi = __half22float2(*reinterpret_cast<const __half2*>(&qf[nt][0][s][h]));
                qf[nt][1][s][h] = half2_bits(u - hi.x, v - hi.y);
              }
            }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            qs[nt][e] = __shfl_sync(0xffffffffu, down, (2 * j + e) * 4) * p.scale;
            m[nt][e] = mw[nt][e] = NONE;
            l[nt][e] = 0.f;
          }
#pragma unroll
          for (int i = 0; i < DP / 16; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[nt][i][e] = 0.f;
        }
      }

      cp_wait<Sh::STAGES - 1>();
      __syncwarp();
      const char* st = ring + stage * Sh::STAGE;
      const float* sc = reinterpret_cast<const float*>(st + Sh::T * DP * 2);
      const unsigned mask = *reinterpret_cast<const unsigned*>(sc + 2 * Sh::T);
      float s[Sh::MT][NT][4];
#pragma unroll
      for (int mt = 0; mt < Sh::MT; ++mt) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[mt][nt][e] = 0.f;
#pragma unroll
        for (int i = 0; i < Sh::NK; ++i) {
          const uint4 u = *reinterpret_cast<const uint4*>(st + (mt * 2 * Sh::NK + i) * 512 + lane * 16);
          const uint4 v = *reinterpret_cast<const uint4*>(st + ((mt * 2 + 1) * Sh::NK + i) * 512 + lane * 16);
          const unsigned uw[4] = {u.x, u.y, u.z, u.w}, vw[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const unsigned a0 = cvt_e4m3x2((unsigned short)uw[k]), a2 = cvt_e4m3x2((unsigned short)(uw[k] >> 16));
            const unsigned a1 = cvt_e4m3x2((unsigned short)vw[k]), a3 = cvt_e4m3x2((unsigned short)(vw[k] >> 16));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int t = 0; t < TERMS; ++t)
                mma16816(s[mt][nt], a0, a1, a2, a3, qf[nt][t][4 * i + k][0], qf[nt][t][4 * i + k][1]);
          }
        }
      }

      // scores of tokens 16 mt + 8 r + g (masked: -infinity, the scales 0)
      float sv[Sh::MT][2];
      float top[NT][2], topw[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) top[nt][e] = topw[nt][e] = NONE;
#pragma unroll
      for (int mt = 0; mt < Sh::MT; ++mt)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int k = 16 * mt + 8 * r + g;
          const bool ok = mask >> k & 1;
          const float ks = kv_scale(sc[k]);
          sv[mt][r] = kv_scale(sc[Sh::T + k]);
          const float lsv = lg2(sv[mt][r]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float& x = s[mt][nt][2 * r + e];
              x = ok ? x * (ks * qs[nt][e]) : __int_as_float(0xff800000);
              top[nt][e] = fmaxf(top[nt][e], x);
              topw[nt][e] = fmaxf(topw[nt][e], x + lsv);
            }
        }
      bool grew = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int k = 4; k < 32; k <<= 1) {
            top[nt][e] = fmaxf(top[nt][e], __shfl_xor_sync(0xffffffffu, top[nt][e], k));
            topw[nt][e] = fmaxf(topw[nt][e], __shfl_xor_sync(0xffffffffu, topw[nt][e], k));
          }
          grew |= top[nt][e] > m[nt][e] || topw[nt][e] > mw[nt][e];
        }
      if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float f[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float mn = fmaxf(m[nt][e], top[nt][e]), mwn = fmaxf(mw[nt][e], topw[nt][e]);
            l[nt][e] *= ex2(m[nt][e] - mn);
            f[e] = ex2(mw[nt][e] - mwn);
            m[nt][e] = mn;
            mw[nt][e] = mwn;
          }
#pragma unroll
          for (int i = 0; i < DP / 16; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[nt][i][e] *= f[e & 1];
        }
      }
      float up[NT][2];   // 2^(m - mw + 15); bounded where all values are zeros
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) up[nt][e] = ex2(fminf(m[nt][e] - mw[nt][e] + 15.f, 126.f));
      unsigned pb[Sh::MT][NT][TERMS][2];
#pragma unroll
      for (int mt = 0; mt < Sh::MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float w[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float pr = ex2(s[mt][nt][2 * r + e] - m[nt][e]);
              l[nt][e] += pr;
              w[e] = pr * up[nt][e] * sv[mt][r];
            }
            const unsigned hi = half2_bits(w[0], w[1]);
            pb[mt][nt][0][r] = transposed8x8(hi);
            if constexpr (TERMS == 2) {
              const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&hi));
              pb[mt][nt][1][r] = transposed8x8(half2_bits(w[0] - h.x, w[1] - h.y));
            }
          }

#pragma unroll
      for (int mt = 0; mt < Sh::MT; ++mt)
#pragma unroll
        for (int i = 0; i < Sh::NV; ++i) {
          unsigned w[4][Sh::VB / 4];   // tokens 2j, 2j + 1, 2j + 8, 2j + 9: VB adjacent columns
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const char* src = st + Sh::T * DP + ((mt * 4 + r) * Sh::NV + i) * (32 * Sh::VB) + lane * Sh::VB;
            if constexpr (Sh::VB == 16) {
              const uint4 u = *reinterpret_cast<const uint4*>(src);
              w[r][0] = u.x, w[r][1] = u.y, w[r][2] = u.z, w[r][3] = u.w;
            } else {
              const uint2 u = *reinterpret_cast<const uint2*>(src);
              w[r][0] = u.x, w[r][1] = u.y;
            }
          }
#pragma unroll
          for (int k = 0; k < Sh::VB / 2; ++k) {
            unsigned x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = cvt_e4m3x2((unsigned short)(w[r][k / 2] >> (16 * (k & 1))));
            const unsigned a0 = __byte_perm(x[0], x[1], 0x5410), a1 = __byte_perm(x[0], x[1], 0x7632);
            const unsigned a2 = __byte_perm(x[2], x[3], 0x5410), a3 = __byte_perm(x[2], x[3], 0x7632);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int t = 0; t < TERMS; ++t)
                mma16816(o[nt][i * (Sh::VB / 2) + k], a0, a1, a2, a3, pb[mt][nt][t][0], pb[mt][nt][t][1]);
          }
        }
      __syncwarp();   // the stage's scales and mask have been read
      issue();
      stage = stage + 1 == Sh::STAGES ? 0 : stage + 1;
      --to_do;

      const bool ends = at.step + 1 == at.steps;
      if (!ends && to_do > 0) {
        ++at.step;
        continue;
      }
      // the unit, or this warp's part of it, is over
      const int head = at.unit / p.tiles, tile = at.unit - head * p.tiles;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int k = 4; k < 32; k <<= 1) l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], k);
      if (begun && ends) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int qi = tile * Sh::NQ + nt * 8 + 2 * j + e;
            if (qi >= p.group) continue;
            const int qh = head * p.group + qi;
            T* out = reinterpret_cast<T*>(a.out) + at.b * a.ldo + (long long)qh * dim;
            const float f = closing(m[nt][e], l[nt][e], mw[nt][e]);
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) store_row(out, p.pairs, DP / 8 * g + 2 * i, dim, o[nt][i][e] * f, o[nt][i][2 + e] * f);
            if (a.lse && g == 0) a.lse[(long long)at.b * a.q_heads + qh] = lse_of(m[nt][e], l[nt][e]);
          }
      } else {
        const int which = begun;   // the first place: of a unit that began before this warp
        float* part = which ? part1 : part0;
        if (which) {
          cp_wait<0>();   // (nothing is in flight any more: the ring is free)
          __syncwarp();
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float* row = part + (nt * 8 + 2 * j + e) * DP;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i)
              *reinterpret_cast<float2*>(row + DP / 8 * g + 2 * i) = make_float2(o[nt][i][e], o[nt][i][2 + e]);
            if (g == 0)
              *reinterpret_cast<float4*>(part + Sh::NQ * DP + 4 * (nt * 8 + 2 * j + e)) = make_float4(m[nt][e], l[nt][e], mw[nt][e], 0.f);
          }
        if (lane == 0) {
          part_unit[warp][which][0] = at.b;
          part_unit[warp][which][1] = at.unit;
          if (!which) part_ends[warp] = ends;
        }
      }
      begun = 1;
      fresh = true;
      if (to_do > 0) {
        if (ends) next_unit<Sh::T>(c, a.window, units, at);
      }
    }
  }
  __syncthreads();

  // Units of several warps of this block: chain 0 is one that began before the block (warp 0 has
  // its first step here), chain w + 1 the one that warp w began and did not end.
  float* ws = reinterpret_cast<float*>(a.ws) + (long long)blockIdx.x * 2 * Sh::PART;
  int* meta = reinterpret_cast<int*>(reinterpret_cast<float*>(a.ws) + (long long)gridDim.x * 2 * Sh::PART) + 4 * blockIdx.x;
  bool opened = false;   // a unit goes on in the next blocks
  for (int chain = 0; chain <= WARPS; ++chain) {
    const int w = chain ? chain - 1 : 0, k0 = chain ? 1 : 0;
    const int b = part_unit[w][k0][0];
    if (b < 0) continue;
    const int unit = part_unit[w][k0][1];
    int n = 1;   // warps that it goes over, some of them without steps
    bool ends = k0 ? false : part_ends[w];
    while (!ends && w + n < WARPS) {
      if (part_unit[w + n][0][0] == b && part_unit[w + n][0][1] == unit) ends = part_ends[w + n];
      else if (part_unit[w + n][0][0] >= 0) break;
      ++n;
    }
    const int head = unit / p.tiles, tile = unit - head * p.tiles;
    for (int x = threadIdx.x; x < Sh::NQ * (DP / 4); x += 32 * WARPS) {
      const int q = x / (DP / 4), d = 4 * (x - q * (DP / 4)), qi = tile * Sh::NQ + q;
      if (qi >= p.group) continue;
      float4 sum = make_float4(0, 0, 0, 0);
      float m = NONE, mw = NONE, l = 0.f;
      for (int k = 0; k < n; ++k) {
        const int kind = k ? 0 : k0;
        if (part_unit[w + k][kind][0] != b || part_unit[w + k][kind][1] != unit) continue;   // a warp without steps
        const float* part = kind ? reinterpret_cast<const float*>(smem + (w + k) * Sh::RING)
                                 : reinterpret_cast<const float*>(smem + WARPS * Sh::RING) + (w + k) * Sh::PART;
        const float4 st = *reinterpret_cast<const float4*>(part + Sh::NQ * DP + 4 * q);
        const float4 v = *reinterpret_cast<const float4*>(part + q * DP + d);
        const float mn = fmaxf(m, st.x), mwn = fmaxf(mw, st.z), f = ex2(mw - mwn), fk = ex2(st.z - mwn);
        l = l * ex2(m - mn) + st.y * ex2(st.x - mn);
        sum = make_float4(sum.x * f + v.x * fk, sum.y * f + v.y * fk, sum.z * f + v.z * fk, sum.w * f + v.w * fk);
        m = mn;
        mw = mwn;
      }
      if (chain && ends) {
        const int qh = head * p.group + qi;
        T* out = reinterpret_cast<T*>(a.out) + b * a.ldo + (long long)qh * dim;
        const float f = closing(m, l, mw);
        store_row(out, p.pairs, d, dim, sum.x * f, sum.y * f);
        store_row(out, p.pairs, d + 2, dim, sum.z * f, sum.w * f);
        if (a.lse && d == 0) a.lse[(long long)b * a.q_heads + qh] = lse_of(m, l);
      } else {
        float* to = ws + (chain ? Sh::PART : 0);
        *reinterpret_cast<float4*>(to + q * DP + d) = sum;
        if (d == 0) *reinterpret_cast<float4*>(to + Sh::NQ * DP + 4 * q) = make_float4(m, l, mw, 0.f);
      }
    }
    if (chain && !ends) {
      opened = true;
      if (threadIdx.x == 0) meta[0] = b, meta[1] = unit;
    }
  }
  if (!p.whole && threadIdx.x == 0) {
    int n = 0;   // blocks that the opened unit goes on in
    if (opened) {
      // the steps up to its last one, and the block that has that one: the last k with
      // total * k / blocks < those steps
      const Spot s = locate<Sh::T>(c, a.window, units, before, c1 - 1);
      const long long upto = c1 + (s.steps - 1 - s.step);
      n = (int)((upto * blocks + total - 1) / total - 1 - blockIdx.x);
    }
    meta[2] = n;
  }
}

// Units of several blocks: block (i, q) joins query q of the unit that block i of the first kernel
// began, over the parts in the line's order, four at a time side by side.
template <class T, int DP, int NT>
__global__ void __launch_bounds__(DP) k_kv_join(const __grid_constant__ KvCache c, const __grid_constant__ KvAttnArgs a,
                                                const __grid_constant__ Plan p) {
  typedef Shape<DP, NT> Sh;
  __shared__ float4 sums[4][DP / 4];
  __shared__ float st[4][3];
  const int q = blockIdx.y, i = blockIdx.x, k0 = threadIdx.x / (DP / 4), d4 = threadIdx.x % (DP / 4);
  pdl_trigger();
  pdl_wait();
  const float* ws = reinterpret_cast<const float*>(a.ws);
  const int* meta = reinterpret_cast<const int*>(ws + (long long)gridDim.x * 2 * Sh::PART) + 4 * i;
  const int n = meta[2];
  if (n == 0) return;
  const int b = meta[0], unit = meta[1], head = unit / p.tiles, qi = (unit - head * p.tiles) * Sh::NQ + q;
  if (qi >= p.group) return;
  float4 sum = make_float4(0, 0, 0, 0);
  float m = NONE, mw = NONE, l = 0.f;
  auto add = [&](float4 v, float vm, float vl, float vmw) {
    const float mn = fmaxf(m, vm), mwn = fmaxf(mw, vmw), f = ex2(mw - mwn), fk = ex2(vmw - mwn);
    l = l * ex2(m - mn) + vl * ex2(vm - mn);
    sum = make_float4(sum.x * f + v.x * fk, sum.y * f + v.y * fk, sum.z * f + v.z * fk, sum.w * f + v.w * fk);
    m = mn;
    mw = mwn;
  };
#pragma unroll 4
  for (int k = k0; k <= n; k += 4) {
    const float* part = ws + (2ll * (i + k) + (k ? 0 : 1)) * Sh::PART;
    const float4 s = *reinterpret_cast<const float4*>(part + Sh::NQ * DP + 4 * q);
    add(*reinterpret_cast<const float4*>(part + q * DP + 4 * d4), s.x, s.y, s.z);
  }
  sums[k0][d4] = sum;
  if (d4 == 0) st[k0][0] = m, st[k0][1] = l, st[k0][2] = mw;
  __syncthreads();
  if (k0) return;
  for (int k = 1; k < 4; ++k) add(sums[k][d4], st[k][0], st[k][1], st[k][2]);
  const int qh = head * p.group + qi;
  T* out = reinterpret_cast<T*>(a.out) + b * a.ldo + (long long)qh * c.head_dim;
  const float f = closing(m, l, mw);
  store_row(out, p.pairs, 4 * d4, c.head_dim, sum.x * f, sum.y * f);
  store_row(out, p.pairs, 4 * d4 + 2, c.head_dim, sum.z * f, sum.w * f);
  if (a.lse && d4 == 0) a.lse[(long long)b * a.q_heads + qh] = lse_of(m, l);
}

int padded(int dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }
int eights(int dim, int group) { return group > 8 && dim <= 128 ? 2 : 1; }
long long steps_of(int dim, long long tokens) { return (tokens + (dim > 128 ? 15 : 31)) / (dim > 128 ? 16 : 32); }

template <class T, int DP, int NT> cudaError_t attend(const KvCache& c, const KvAttnArgs& a, cudaStream_t s) {
  typedef Shape<DP, NT> Sh;
  static PerDevice<int> sms;
  int dev = 0, n_sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= PerDevice<int>::devices) return cudaErrorNotSupported;
  e = sms.get(dev, &n_sms, [&](int& v) {
    const cudaError_t r = cudaFuncSetAttribute(k_kv_attention<T, DP, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::SMEM);
    return r != cudaSuccess ? r : cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev);
  });
  if (e != cudaSuccess) return e;
  Plan p = {};
  while ((1ll << p.div_s) < c.page_size) ++p.div_s;
  p.div_m = (unsigned)(((1ull << 32) * ((1ull << p.div_s) - c.page_size)) / c.page_size + 1);
  p.group = a.q_heads / c.heads;
  p.tiles = (p.group + Sh::NQ - 1) / Sh::NQ;
  const int es = sizeof(T);
  p.pairs = !((uintptr_t)a.out & (2 * es - 1)) && a.ldo % 2 == 0;
  p.scale = a.scale * 1.4426950408889634f;
  long long tokens = (long long)c.table_pages * c.page_size;
  if (a.window) tokens = std::min(tokens, (long long)a.window);
  const long long units = (long long)c.seqs * c.heads * p.tiles, steps = steps_of(c.head_dim, tokens);
  p.whole = steps <= WHOLE_STEPS;
  // blocks: one to an SM; fewer where there are not two steps to a warp, or no more units
  long long grid = std::min(n_sms, GRID_MAX);
  grid = std::min(grid, p.whole ? units : (units * steps + 2 * WARPS - 1) / (2 * WARPS));
  e = launch_pdl(k_kv_attention<T, DP, NT>, (unsigned)grid, 32 * WARPS, Sh::SMEM, s, c, a, p);
  if (e != cudaSuccess) return e;
  e = launched();
  if (e != cudaSuccess || p.whole) return e;
  e = launch_pdl(k_kv_join<T, DP, NT>, dim3((unsigned)grid, Sh::NQ), DP, 0, s, c, a, p);
  return e != cudaSuccess ? e : launched();
}
template <class T> cudaError_t attend(const KvCache& c, const KvAttnArgs& a, cudaStream_t s) {
  const bool two = eights(c.head_dim, a.q_heads / c.heads) == 2;
  switch (padded(c.head_dim)) {
    case 64: return two ? attend<T, 64, 2>(c, a, s) : attend<T, 64, 1>(c, a, s);
    case 128: return two ? attend<T, 128, 2>(c, a, s) : attend<T, 128, 1>(c, a, s);
    default: return attend<T, 256, 1>(c, a, s);
  }
}

}  // namespace

size_t kv_attention_workspace(int seqs, int q_heads, int heads, int dim, long long tokens) {
  (void)seqs;
  if (steps_of(dim, tokens) <= WHOLE_STEPS) return 0;
  return GRID_MAX * (2 * 8 * (size_t)eights(dim, q_heads / heads) * (padded(dim) + 4) * 4 + 16);
}

cudaError_t launch_kv_attention(DType dt, const KvCache& c, const KvAttnArgs& a, cudaStream_t s) {
  return dt == F32 ? attend<float>(c, a, s) : attend<bf16>(c, a, s);
}

}  // namespace ff
