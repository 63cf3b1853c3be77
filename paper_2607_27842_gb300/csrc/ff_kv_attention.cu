// Attention of one new token of each sequence over the 8-bit key-value cache
// (formulas: featfix_op_kv_attention).  Bound by memory: every cached byte that a token sees is read
// once for up to 16 query heads of its key head (8 of more than 128 columns).  More are units of their
// own, which read it again: 64 x 8192 tokens, 8 key heads of 128 with 16 query heads each 266 us, with 32 486.
//
// The work is a line of steps: a unit is one key head of one sequence with up to 8 or 16 of
// its query heads, a step T of its tokens.  Units of a sequence whose number divides the
// warps go together, one to a warp (or to several, which share out the steps): their places are
// adjacent in memory, as are their scales.  The line has the steps of one such group, of the
// sequence's next one, then of the next sequence's; every block takes an equal stretch of it,
// whatever the lengths are, and every warp goes over its own on its own.  Tokens come by
// asynchronous copies a step or two ahead, eight lanes to 128 adjacent bytes, into a ring that only
// this warp knows; e4m3 becomes fp16 in registers, exactly; products are mma.sync m16n8k16 with
// tokens or columns as the 16 and query heads as the 8, because a token's few query heads would
// fill 4 of tcgen05's 128 rows, and the products are far from a bound here.
//
//   S^T[token, query] = K Q^T,   O^T[column, query] += V^T P^T
//
// Sums over any index may go in any order as long as both factors agree on it: lane (g, j) =
// (lane / 4, lane % 4) holds 16 adjacent columns of keys g and g + 8, and for the second
// product 16 adjacent columns of values 2j, 2j + 1, 2j + 8, 2j + 9, whole 16-byte vectors in the
// order of memory.  P^T turns from the one's result to the other's operand in movmatrix.
//
// Softmax with a running maximum m of the scores x (in powers of two).  Its sum l takes p = exp2(x - m) in
// fp32.  The weights p * scale_v go to fp16, times the power of two that brings the largest of them so far,
// w, to 2^14 .. 2^15: they use all of fp16's range whatever the scales are, and weights 2^-28 below the
// largest still have 11 bits.  w is kept relative to m, as l is: a sum x + log2(scale_v) would lose the
// scale in the rounding of large x (from 2^24 on more than a factor of two, past fp16's largest number).
//
// Bits.  Scores, m, l, w and all sums are fp32.  e4m3 is exact in fp16, and so are bf16 queries (but for elements
// 2^-29 below the largest of a head): one term.  fp32 queries and all weights are two fp16 terms, 22 bits: errors
// against 64 bits are 7.0e-7 in fp32 (48 x 700 tokens), and third terms leave them there (7.1e-7, and 16 to 20% more
// time for the queries'), as they come from the exponential, the scores' rounding and the products' sums.  Weights in one term
// (11 bits) made 5% of bf16 results round the other way than fp32 weights do, where two make 0.1%: 64 x 8192
// tokens 192.4 and 190.8 us, 64 ragged 103.7 and 104.2, 1 x 257 7.07 and 7.25, 4096 x 32 115 and 119, heads of 64 and
// 256 3% more.
//
// A stretch begins and ends within units.  What belongs to one unit of several warps meets in
// shared memory at the end, and of several blocks in the workspace, which a second
// kernel adds in the line's order: no atomics, the same bits every time.
//
// Measured, heads of 128 in bf16: 64 sequences of 8192 tokens, 32 + 8 heads, 185 us, 6.0 TB/s; 64 of 4096
// with fp32 queries 108 us, 5.1 TB/s, where the queries' two terms double the first product; 1 x 131072, 16 + 4
// heads, 34 us, of which the loop takes 21 (6.7 TB/s) and start, the joins of warps and the second kernel 13;
// 1 x 257 7 us, a chain of waits.
#include "ff_kv8.cuh"
#include "ff_host.h"

#include <cuda_fp16.h>

#include <algorithm>
#include <type_traits>

namespace ff {

namespace {

constexpr int GRID_MAX = 160;      // blocks that the workspace has room for
constexpr float NONE = -3.0e38f;   // maximum of nothing
// Blocks take whole units, and there is no second kernel, where units are short: at most WHOLE_STEPS steps
// (1 x 1000 tokens of 16 + 4 heads 11.1 us so and 13.6 shared out, 1 x 2000 17.3 and 14.0), and a block's
// fit its warps (200 x 1000 tokens of 32 + 8 heads 73 and 86 us) or have WHOLE_SUM steps in all (256 x 256
// tokens 36.3 and 41.6, 256 x 1000 106 and 104, 4096 x 32 130 and 115).  The 152 are this rule's, not the call's GPU's: a
// workspace is asked for without one, and both sides have to agree.
constexpr int WHOLE_STEPS = 32, WHOLE_SUM = 160, SMS = 152;
bool whole_units(long long units, long long steps, int warps) {
  return steps <= WHOLE_STEPS && (units <= (long long)SMS * warps || units * steps <= SMS * WHOLE_SUM);
}

// Shapes of a variant: columns of a head rounded up to DP, NT times 8 query heads.
template <class E, int DP, int NT> struct Shape {
  // warps of a block: as many as have the registers for their sums and queries.  A spilled register
  // in the loop goes through the 20 KB of L1 that the rings leave: 64 x 8192 tokens took 221 us with
  // 16 warps of 128 registers (80 bytes spilled), 189 with 12 of 168, 206 with 8; 64 x 4096 in fp32 123 with
  // 8 and 109 with 12, though 92 bytes spill.
  static constexpr int WARPS = NT > 1 || DP == 256 ? 8 : DP == 64 && sizeof(E) == 2 ? 16 : 12;
  static constexpr int MT = DP == 256 ? 1 : 2;                 // groups of 16 tokens in a step
  static constexpr int T = 16 * MT;
  static constexpr int STAGES = (DP == 64 ? 2 : 1) * (WARPS > 8 ? 1 : 2);
  static constexpr int NK = DP / 64;                           // 16-byte vectors of a key to a lane
  static constexpr int ROWS = 512 / DP;                        // tokens of a copy by all lanes
  static constexpr int VB = DP >= 128 ? 16 : 8;                // bytes of a value's vector
  static constexpr int NV = DP / 8 / VB;
  static constexpr int STAGE = T * DP * 2 + T * 8 + 16;        // keys, values, scales, mask
  static constexpr int RING = STAGE * STAGES;                  // of a warp
  static constexpr int NQ = 8 * NT;
  static constexpr int PART = NQ * (DP + 4);                   // floats: sums, then m, l, w of each query
  static constexpr int SMEM = WARPS * (RING + PART * 4);
  static_assert(PART * 4 <= RING, "the second partial result lies in the ring");
  static_assert(STAGE % 16 == 0 && PART % 4 == 0, "whole vectors");
};

struct Plan {
  Div page, split_by, tiles_by, blocks_by, together_by, groups_by;   // page_size, split, ..., the grid
  int group, tiles;        // query heads of a key head, units that share them
  int together, split, groups;   // units that go together, warps to each of them, groups of a sequence
  int units;               // of all sequences, where whole is 2 (and a group is a unit)
  int join_queries, grid;  // queries to a block of the second kernel, blocks of the first
  int whole;               // blocks take whole units; 2: the same number each, at most one to a warp
  int pairs, vectors;      // results may be stored in pairs, queries loaded four at a time
  float scale;             // softmax scale times log2(e)
  // strides of page and slot of keys and values in units of 2^shift bytes, by which every place's
  // offset fits 32 bits; of their scales in floats
  unsigned k_unit[2], v_unit[2], ks[2], vs[2];
  unsigned k_bytes, v_bytes;   // 2^shift
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
// Weights up to w, of exponent e = top_exp(w), are below 2^15 times raised(e) = 2^(141 - e); lowered(e) is
// 1 / raised(e).  (Weights all below 2^-111 come from scales that no written token has.)
__device__ __forceinline__ int top_exp(float w) { return max(15, (int)(__float_as_uint(w) >> 23)); }
__device__ __forceinline__ float raised(int e) { return __int_as_float((268 - e) << 23); }
__device__ __forceinline__ float lowered(int e) { return __int_as_float((e - 14) << 23); }
// 2^(from - to): turns sums of weights raised by `from` into such raised by `to`.  (Past 2^127 the factor that it
// goes with has become 0; below 2^-126 nothing is left of the sums beside weights of 2^14.)
__device__ __forceinline__ float moved(int from, int to) { return __int_as_float((max(-126, min(127, from - to)) + 127) << 23); }
__device__ __forceinline__ unsigned half2_bits(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const unsigned*>(&h);
}
__device__ __forceinline__ void cp_async16s(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// Where the 16 bytes from column 16 * chunk of token `row` lie in a stage's keys or values: lines of
// 128 bytes (half a token, a token or two) whose vectors change places from line to line, so
// that neither products' reads (eight lanes: two tokens by four vectors for keys, four tokens
// by two for values) have two lanes on one bank.
template <int DP, int T> __device__ __forceinline__ int place(int row, int chunk) {
  if constexpr (DP == 64) {
    const int line = row >> 1;
    return line * 128 + (((row & 1) * 4 + chunk) ^ (2 * (line & 3))) * 16;
  } else {
    return ((chunk >> 3) * T + row) * 128 + ((chunk & 7) ^ ((row & 6) ^ (row & 1) * 4)) * 16;
  }
}
// First of the two columns of a value that lane group g has in its i-th product.
template <int DP> __device__ __forceinline__ int column(int g, int i) {
  return DP == 256 ? 128 * (i >> 3) + 16 * g + 2 * (i & 7) : DP / 8 * g + 2 * i;
}

// Lengths and page numbers may change while the kernel runs.  Results mean nothing then, but nothing may be
// read or written out of range, nor lanes of a warp part.  So what a warp does by a length goes by lane 0's
// load of it, a page number is one load, which the compiler may not repeat, and what either leads to is
// bounded.  (4096 sequences of 32 tokens 114.4 -> 115.3 us.)
__device__ __forceinline__ int shared_by_all(int v) { return __shfl_sync(0xffffffffu, v, 0); }
__device__ __forceinline__ int once(const int* p) {
  int v;
  asm volatile("ld.global.s32 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}

// Tokens that sequence b's new token sees.
struct Seen {
  int first, end;
};
__device__ __forceinline__ Seen seen_of(int len, int window) { return {window && len > window ? len - window : 0, len}; }
__device__ __forceinline__ int len_of(const KvCache& c, int b) { return kv_len(c, c.lens[b]); }
// (by a whole warp)
__device__ __forceinline__ Seen seen(const KvCache& c, int window, int b) { return seen_of(shared_by_all(len_of(c, b)), window); }

// Where a step of the line is: sequence, unit (as locate() finds it: group of units), step, and how
// many steps the sequence has.
struct Spot {
  int b, unit, step, steps;
};
template <int T> __device__ __forceinline__ int steps_of_lane(const KvCache& c, int window, int b) {
  const Seen s = seen_of(len_of(c, b), window);
  return (s.end - s.first + T - 1) / T;
}
template <int T> __device__ __forceinline__ int steps_seen(const KvCache& c, int window, int b) {   // (by a whole warp)
  return shared_by_all(steps_of_lane<T>(c, window, b));
}

// a / b for a >= 0, b > 0
__device__ __noinline__ long long quot64(long long a, long long b) { return a / b; }
__device__ __forceinline__ long long quot(long long a, long long b) {
  return (a | b) >> 31 ? quot64(a, b) : (int)((unsigned)a / (unsigned)b);
}
__device__ __forceinline__ long long quot(long long a, long long b, const Div& by) {
  return a >> 31 ? quot64(a, b) : by.of((unsigned)a);
}

// The line, as every warp finds it on its own: a lane has a share of adjacent sequences.
struct Line {
  long long before, total;   // steps of the shares before this lane's, and of all
  int per;                   // sequences to a share
};
template <int T> __device__ __forceinline__ Line line_up(const KvCache& c, int window, int groups) {
  const int lane = threadIdx.x & 31, per = (c.seqs + 31) / 32;
  long long n = 0;
#pragma unroll 4
  for (int i = 0; i < per; ++i)
    if (lane * per + i < c.seqs) n += steps_of_lane<T>(c, window, lane * per + i);
  n *= groups;
  long long sum = n;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += v;
  }
  return {sum - n, __shfl_sync(0xffffffffu, sum, 31), per};
}
// The spot of step `at` of the line (below its length), by a whole warp.
template <int T> __device__ __noinline__ Spot locate(const KvCache& c, int window, int groups, Line line, long long at) {
  // the last share that starts at or before `at`
  const int lo = __popc(__ballot_sync(0xffffffffu, line.before <= at)) - 1;
  at -= __shfl_sync(0xffffffffu, line.before, lo);
  for (int b = lo * line.per; b < c.seqs; ++b) {
    const int steps = steps_seen<T>(c, window, b);
    if (at < (long long)steps * groups) {
      const int group = groups == 1 ? 0 : (int)quot(at, steps);
      return {b, group, (int)(at - (long long)group * steps), steps};
    }
    at -= (long long)steps * groups;
  }
  return {c.seqs - 1, 0, 0, 1};   // (lengths that change meanwhile: no address out of range)
}

// The warp's next unit that has steps: of the sequence's next group, or of the next sequence.
// `of` follows: what its sequence's new token sees.
template <int T> __device__ __forceinline__ void next_unit(const KvCache& c, const Plan& p, int window, int u, Spot& s, Seen& of) {
  s.step = 0;
  s.unit += p.together;
  if (s.unit < c.heads * p.tiles) return;
  s.unit = u;
  do {
    if (s.b + 1 >= c.seqs) return;   // (as above: the line has an end before)
    of = seen(c, window, ++s.b);
    s.steps = (of.end - of.first + T - 1) / T;
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
// By which sums become results; 0 for a row of no tokens.
__device__ __forceinline__ float closing(float l, float w) { return l == 0.f ? 0.f : lowered(top_exp(w)) / l; }
__device__ __forceinline__ float lse_of(float m, float l) {
  return l == 0.f ? __int_as_float(0xff800000) : (m + log2f(l)) * 0.69314718055994531f;
}

template <class T, int DP, int NT>
__global__ void __launch_bounds__(32 * Shape<T, DP, NT>::WARPS, 1) k_kv_attention(const __grid_constant__ KvCache c,
                                                                 const __grid_constant__ KvAttnArgs a,
                                                                 const __grid_constant__ Plan p) {
  typedef Shape<T, DP, NT> Sh;
  constexpr int WARPS = Sh::WARPS, TERMS = sizeof(T) == 4 ? 2 : 1;   // fp16 terms of queries
  extern __shared__ __align__(16) char smem[];
  // partial results of the block's units, in the line's order: what a warp has of a unit that began
  // before its stretch, then of one that goes on behind it
  __shared__ int2 part_of[2 * WARPS];             // sequence (-1: none), 2 * unit + whether its last step is in
  __shared__ long long part_upto[WARPS];          // the line's steps up to the end of a unit that goes on
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, j = lane & 3;
  const int dim = c.head_dim;
  if (lane < 2) part_of[2 * warp + lane] = make_int2(-1, 0);
  __syncwarp();
  pdl_trigger();
  pdl_wait();

  // This warp's steps of the line: w1 - w0 from `at` on, in a block's c0 .. c1.
  const int sp = p.together_by.of(warp), u = warp - sp * p.together, groups = p.groups;
  Spot at;
  long long w0, w1, c1 = 0, total = 1, blocks = 1;
  auto stretch = [&](long long c0, long long n) {
    // (rounded up: the first warp of a unit has steps where any has)
    w0 = c0 + (sp < p.split ? quot(n * sp + p.split - 1, p.split, p.split_by) : n);
    w1 = c0 + (sp < p.split ? quot(n * (sp + 1) + p.split - 1, p.split, p.split_by) : n);
  };
  if (p.whole == 2) {   // some units to a block, as many warps to each
    // (to the kernel these warps go together; the units need not be of one sequence)
    const long long unit = (long long)blockIdx.x * p.together + u;
    const int b = unit < p.units ? p.groups_by.of((unsigned)unit) : 0;
    const int steps = unit < p.units ? steps_seen<Sh::T>(c, a.window, b) : 0;
    stretch(0, steps);
    at = {b, (int)unit - b * groups, (int)w0, steps};
  } else {
    const Line line = line_up<Sh::T>(c, a.window, groups);
    total = line.total;
    // blocks that have a share: with a step to every warp
    blocks = p.whole ? gridDim.x : max(1ll, min((long long)gridDim.x, quot(total + p.split - 1, p.split, p.split_by)));
    auto edge = [&](long long i) {   // of block i: its first step of the line
      long long e = i >= blocks ? total : blocks == gridDim.x ? quot(total * i, blocks, p.blocks_by) : quot(total * i, blocks);
      if (p.whole && e < total) {
        const Spot s = locate<Sh::T>(c, a.window, groups, line, e);
        if (s.step) e += s.steps - s.step;
      }
      return e;
    };
    const long long c0 = edge(blockIdx.x);
    c1 = edge(blockIdx.x + 1ll);
    stretch(c0, c1 - c0);
    if (w0 < w1) {
      at = locate<Sh::T>(c, a.window, groups, line, w0);
      at.unit = at.unit * p.together + u;
    }
  }

  char* ring = smem + warp * Sh::RING;
  float* part0 = reinterpret_cast<float*>(smem + WARPS * Sh::RING) + warp * Sh::PART;
  float* part1 = reinterpret_cast<float*>(ring);
  const uint32_t ring_s = (uint32_t)__cvta_generic_to_shared(ring);

  if (w0 < w1) {
    Spot in = at;
    int to_issue = (int)min((long long)0x7fffffff, w1 - w0), to_do = to_issue;
    Seen in_seen = seen(c, a.window, in.b);

    // Page of this lane's token of the step at `in`, looked up one step before its copies.
    auto token = [&] { return in_seen.first + in.step * Sh::T + (lane & (Sh::T - 1)); };
    auto page_of = [&](int t) { return p.page.of((unsigned)t); };
    auto look_up = [&] {
      const int t = token();
      return (unsigned)t < (unsigned)in_seen.end ? once(c.table + in.b * c.ld_table + page_of(t)) : -1;
    };
    int entry = look_up();
    int stage_in = 0;
    // this lane's part of every copy: 16 bytes of the token at lane / (DP / 16) behind the copy's first
    const int col = 16 * (lane % (DP / 16)), sub = lane / (DP / 16), n_col = min(16, max(0, dim - col));
    const char *kb, *vb;   // of the unit's key head
    const float *ksb, *vsb;
    auto heads_of = [&](int unit) {
      const int head = p.tiles_by.of(unit);
      kb = reinterpret_cast<const char*>(c.k) + head * c.k_stride[2];
      vb = reinterpret_cast<const char*>(c.v) + head * c.v_stride[2];
      ksb = c.k_scale + head * c.k_scale_stride[2];
      vsb = c.v_scale + head * c.v_scale_stride[2];
    };
    heads_of(in.unit);
    unsigned in_page = 0, in_slot = 0, in_mask = 0;
    float ks_in = 0.f, vs_in = 0.f;   // scales of this lane's token of the last step that was issued, and
    // where they go when they have come (before the first: where no copy goes, whose order with these stores is open)
    char* scales_to = ring + Sh::T * DP * 2 + 4 * lane;
    // Copies of a step's tokens from base + unit * (their offsets) to dst; `all`: no token of it is masked.
    auto copy = [&](auto all, uint32_t dst, const char* base, unsigned unit, unsigned at) {
      base += n_col ? col : 0;
#pragma unroll
      for (int i = 0; i < Sh::T / Sh::ROWS; ++i) {
        const int row = Sh::ROWS * i + sub;
        const char* src = base + (unsigned long long)__shfl_sync(0xffffffffu, at, row) * unit;
        const uint32_t to = dst + place<DP, Sh::T>(row, lane % (DP / 16));
        cp_async16s(to, src, all || (in_mask >> row & 1) ? n_col : 0);
      }
    };
    // The next step's keys, then its values, each a group of copies on its own (an empty one
    // behind the last step keeps the count).
    auto issue_keys = [&] {
      if (to_issue > 0) {
        const int t = token();
        const bool there = (unsigned)entry < (unsigned)c.pages && (unsigned)t < (unsigned)in_seen.end;
        in_page = there ? entry : 0;
        in_slot = there ? t - page_of(t) * c.page_size : 0;
        in_mask = __ballot_sync(0xffffffffu, there);
        const uint32_t st = ring_s + stage_in * Sh::STAGE;
        const unsigned kat = in_page * p.k_unit[0] + in_slot * p.k_unit[1];
        if (in_mask == 0xffffffffu) copy(std::true_type(), st, kb, p.k_bytes, kat);
        else copy(std::false_type(), st, kb, p.k_bytes, kat);
        ks_in = vs_in = 0.f;
        scales_to = ring + stage_in * Sh::STAGE + Sh::T * DP * 2 + 4 * lane;
        if (there) {
          ks_in = ksb[(unsigned long long)in_page * p.ks[0] + (unsigned long long)in_slot * p.ks[1]];
          vs_in = vsb[(unsigned long long)in_page * p.vs[0] + (unsigned long long)in_slot * p.vs[1]];
        }
        if (lane == 0) *reinterpret_cast<unsigned*>(ring + stage_in * Sh::STAGE + Sh::T * DP * 2 + Sh::T * 8) = in_mask;
      }
      cp_commit();
    };
    auto issue_values = [&] {
      if (to_issue > 0) {
        const uint32_t st = ring_s + stage_in * Sh::STAGE + Sh::T * DP;
        const unsigned vat = in_page * p.v_unit[0] + in_slot * p.v_unit[1];
        if (in_mask == 0xffffffffu) copy(std::true_type(), st, vb, p.v_bytes, vat);
        else copy(std::false_type(), st, vb, p.v_bytes, vat);
        stage_in = stage_in + 1 == Sh::STAGES ? 0 : stage_in + 1;
        if (--to_issue > 0) {
          if (++in.step == in.steps) {
            next_unit<Sh::T>(c, p, a.window, u, in, in_seen);
            heads_of(in.unit);
          }
          entry = look_up();
        }
      }
      cp_commit();
    };
    unsigned qf[NT][TERMS][DP / 16][2];
    float qs[NT][2];                         // of queries 2j, 2j + 1: what a product is multiplied by
    float m[NT][2], l[NT][2], w[NT][2], o[NT][DP / 16][4];   // (w: see above)
    // Queries of the unit at `at`, as they are in memory: of query g of the tile four adjacent columns
    // for each 16 of the sum.
    auto load_queries = [&] {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int head = p.tiles_by.of(at.unit), qi = (at.unit - head * p.tiles) * Sh::NQ + nt * 8 + g;
        const T* q = reinterpret_cast<const T*>(a.q) + at.b * a.ldq + (long long)(head * p.group + qi) * dim;
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
          const int col = 16 * (j + 4 * (s / 4)) + 4 * (s % 4);
          const bool in = qi < p.group && col < dim;
          if constexpr (TERMS == 1) {
            uint2 v = make_uint2(0, 0);
            if (in) {
              if (p.vectors) {
                v = *reinterpret_cast<const uint2*>(q + col);
              } else {
                const unsigned short* h = reinterpret_cast<const unsigned short*>(q + col);
                v = make_uint2(h[0] | (unsigned)h[1] << 16, h[2] | (unsigned)h[3] << 16);
              }
            }
            qf[nt][0][s][0] = v.x, qf[nt][0][s][1] = v.y;
          } else {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (in) {
              const unsigned* w = reinterpret_cast<const unsigned*>(q + col);
              v = p.vectors ? *reinterpret_cast<const uint4*>(w) : make_uint4(w[0], w[1], w[2], w[3]);
            }
            qf[nt][0][s][0] = v.x, qf[nt][1][s][0] = v.y, qf[nt][0][s][1] = v.z, qf[nt][1][s][1] = v.w;
          }
        }
      }
    };
    load_queries();
    int stage = 0;
    bool begun = at.step == 0, fresh = true;   // whether this warp has the unit's first step; its queries come next
    // (the first rounds only fill the ring: one copy of the code that does)
    for (int round = -Sh::STAGES; to_do > 0; ++round) {
      const bool on = round >= 0;
      if (lane < Sh::T) {
        *reinterpret_cast<float*>(scales_to) = kv_scale(ks_in);
        *reinterpret_cast<float*>(scales_to + 4 * Sh::T) = kv_scale(vs_in);
      }
      unsigned mask = 0;
      float s[Sh::MT][NT][4];
      if (on) {
      if (fresh) {
        fresh = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          auto raw = [&](int s, int h) {   // columns 2 h, 2 h + 1 of the four
            if constexpr (TERMS == 1) {
              const f32x2 v = bf2u(qf[nt][0][s][h]);
              return make_float2(lo_f(v), hi_f(v));
            } else {
              return make_float2(__uint_as_float(qf[nt][0][s][h]), __uint_as_float(qf[nt][1][s][h]));
            }
          };
          float top = 0.f;
#pragma unroll
          for (int s = 0; s < DP / 16; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) top = max_abs(top, max_abs(raw(s, h).x, raw(s, h).y));
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
              const float2 x = raw(s, h);
              const float u = x.x * up, v = x.y * up;
              qf[nt][0][s][h] = half2_bits(u, v);
              if constexpr (TERMS == 2) {
                const float2 hi = __half22float2(*reinterpret_cast<const __half2*>(&qf[nt][0][s][h]));
                qf[nt][1][s][h] = half2_bits(u - hi.x, v - hi.y);
              }
            }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            qs[nt][e] = __shfl_sync(0xffffffffu, down, (2 * j + e) * 4) * p.scale;
            m[nt][e] = NONE;
            l[nt][e] = w[nt][e] = 0.f;
          }
#pragma unroll
          for (int i = 0; i < DP / 16; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[nt][i][e] = 0.f;
        }
      }

      cp_wait<2 * Sh::STAGES - 1>();
      __syncwarp();
      const char* st = ring + stage * Sh::STAGE;
      const float* sc = reinterpret_cast<const float*>(st + Sh::T * DP * 2);
      mask = *reinterpret_cast<const unsigned*>(sc + 2 * Sh::T);
#pragma unroll
      for (int mt = 0; mt < Sh::MT; ++mt) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[mt][nt][e] = 0.f;
#pragma unroll
        for (int i = 0; i < Sh::NK; ++i) {
          const uint4 u = *reinterpret_cast<const uint4*>(st + place<DP, Sh::T>(16 * mt + g, j + 4 * i));
          const uint4 v = *reinterpret_cast<const uint4*>(st + place<DP, Sh::T>(16 * mt + 8 + g, j + 4 * i));
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

      // scores of tokens 16 mt + 8 r + g (masked: -infinity)
#pragma unroll
      for (int mt = 0; mt < Sh::MT; ++mt)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int k = 16 * mt + 8 * r + g;
          const float ks = sc[k];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float& x = s[mt][nt][2 * r + e];
              x *= ks * qs[nt][e];
              if (mask != 0xffffffffu && !(mask >> k & 1)) x = __int_as_float(0xff800000);
            }
        }
      __syncwarp();   // the stage's keys, their scales and the mask have been read
      }
      issue_keys();
      if (on) {
      cp_wait<2 * Sh::STAGES - 1>();
      __syncwarp();
      const char* st = ring + stage * Sh::STAGE;
      const float* sc = reinterpret_cast<const float*>(st + Sh::T * DP * 2);

      float by[NT][2];   // exp2 of what m grows by, negative
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float top = m[nt][e];
#pragma unroll
          for (int mt = 0; mt < Sh::MT; ++mt) top = fmaxf(top, fmaxf(s[mt][nt][e], s[mt][nt][2 + e]));
#pragma unroll
          for (int k = 4; k < 32; k <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
          by[nt][e] = ex2(m[nt][e] - top);
          m[nt][e] = top;
        }
      // p, its sum, and the weights p * scale_v (of masked tokens 0)
      float topw[NT][2], sum[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) topw[nt][e] = sum[nt][e] = 0.f;
#pragma unroll
      for (int mt = 0; mt < Sh::MT; ++mt)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float sv = sc[Sh::T + 16 * mt + 8 * r + g];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float& x = s[mt][nt][2 * r + e];
              const float pr = ex2(x - m[nt][e]);
              sum[nt][e] += pr;
              x = pr * sv;
              topw[nt][e] = fmaxf(topw[nt][e], x);
            }
        }
      bool grew = false;
      int from[NT][2], to[NT][2];   // exponents that sums and weights are raised by
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int k = 4; k < 32; k <<= 1) topw[nt][e] = fmaxf(topw[nt][e], __shfl_xor_sync(0xffffffffu, topw[nt][e], k));
          from[nt][e] = top_exp(w[nt][e]);
          w[nt][e] = fmaxf(w[nt][e] * by[nt][e], topw[nt][e]);
          to[nt][e] = top_exp(w[nt][e]);
          l[nt][e] = fmaf(l[nt][e], by[nt][e], sum[nt][e]);
          grew |= by[nt][e] != 1.f || from[nt][e] != to[nt][e];
        }
      if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float f[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) f[e] = by[nt][e] * moved(from[nt][e], to[nt][e]);
#pragma unroll
          for (int i = 0; i < DP / 16; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[nt][i][e] *= f[e & 1];
        }
      }
#pragma unroll
      for (int mt = 0; mt < Sh::MT; ++mt) {
        unsigned pb[NT][2][2];   // two fp16 terms of weights
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const float u = s[mt][nt][2 * r] * raised(to[nt][0]), v = s[mt][nt][2 * r + 1] * raised(to[nt][1]);
            const unsigned hi = half2_bits(u, v);
            pb[nt][0][r] = transposed8x8(hi);
            const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&hi));
            pb[nt][1][r] = transposed8x8(half2_bits(u - h.x, v - h.y));
          }
#pragma unroll
        for (int i = 0; i < Sh::NV; ++i) {
          unsigned vw[4][Sh::VB / 4];   // tokens 2j, 2j + 1, 2j + 8, 2j + 9: VB adjacent columns
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int row = 16 * mt + 8 * (r >> 1) + 2 * j + (r & 1), at = column<DP>(g, i * (Sh::VB / 2));
            const char* src = st + Sh::T * DP + place<DP, Sh::T>(row, at / 16) + at % 16;
            if constexpr (Sh::VB == 16) {
              const uint4 u = *reinterpret_cast<const uint4*>(src);
              vw[r][0] = u.x, vw[r][1] = u.y, vw[r][2] = u.z, vw[r][3] = u.w;
            } else {
              const uint2 u = *reinterpret_cast<const uint2*>(src);
              vw[r][0] = u.x, vw[r][1] = u.y;
            }
          }
#pragma unroll
          for (int k = 0; k < Sh::VB / 4; ++k) {
            // bytes of two tokens side by side: a conversion makes a column's pair of tokens
            const unsigned x[2] = {__byte_perm(vw[0][k], vw[1][k], 0x5140), __byte_perm(vw[0][k], vw[1][k], 0x7362)};
            const unsigned y[2] = {__byte_perm(vw[2][k], vw[3][k], 0x5140), __byte_perm(vw[2][k], vw[3][k], 0x7362)};
            unsigned a[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              a[h][0] = cvt_e4m3x2((unsigned short)x[h]), a[h][1] = cvt_e4m3x2((unsigned short)(x[h] >> 16));
              a[h][2] = cvt_e4m3x2((unsigned short)y[h]), a[h][3] = cvt_e4m3x2((unsigned short)(y[h] >> 16));
            }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                  mma16816(o[nt][i * (Sh::VB / 2) + 2 * k + h], a[h][0], a[h][1], a[h][2], a[h][3], pb[nt][t][0], pb[nt][t][1]);
          }
        }
      }
      __syncwarp();   // the stage's values and their scales have been read
      }
      issue_values();
      if (!on) continue;
      stage = stage + 1 == Sh::STAGES ? 0 : stage + 1;
      --to_do;

      const bool ends = at.step + 1 == at.steps;
      if (!ends && to_do > 0) {
        ++at.step;
        continue;
      }
      // the unit, or this warp's part of it, is over
      const int head = p.tiles_by.of(at.unit), tile = at.unit - head * p.tiles;
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
            const float f = closing(l[nt][e], w[nt][e]);
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) store_row(out, p.pairs, column<DP>(g, i), dim, o[nt][i][e] * f, o[nt][i][2 + e] * f);
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
              *reinterpret_cast<float2*>(row + column<DP>(g, i)) = make_float2(o[nt][i][e], o[nt][i][2 + e]);
            if (g == 0)
              *reinterpret_cast<float4*>(part + Sh::NQ * DP + 4 * (nt * 8 + 2 * j + e)) = make_float4(m[nt][e], l[nt][e], w[nt][e], 0.f);
          }
        if (lane == 0) {
          part_of[2 * warp + which] = make_int2(at.b, 2 * at.unit + ends);
          part_upto[warp] = w1 + (at.steps - 1 - at.step);
        }
      }
      begun = true;
      fresh = true;
      if (to_do > 0) {
        Seen of;
        next_unit<Sh::T>(c, p, a.window, u, at, of);
        load_queries();
      }
    }
  }

  // rows of sequences without tokens
  for (int b = blockIdx.x; b < c.seqs; b += gridDim.x) {
    if (steps_of_lane<Sh::T>(c, a.window, b)) continue;
    T* out = reinterpret_cast<T*>(a.out) + b * a.ldo;
    for (int i = threadIdx.x; i < a.q_heads * dim; i += 32 * WARPS) out[i] = from_f<T>(0.f);
    if (a.lse)
      for (int i = threadIdx.x; i < a.q_heads; i += 32 * WARPS) a.lse[(long long)b * a.q_heads + i] = __int_as_float(0xff800000);
  }

  __syncthreads();
  // A warp joins one query of the units that one place of the groups had: lane r holds which unit the
  // r-th of their partial results is of, and the factor that brings it to the unit's maxima; then
  // a lane has four columns.
  const int queries = min(Sh::NQ, p.group), n_parts = 2 * p.split;
  float* ws = reinterpret_cast<float*>(a.ws) + (long long)blockIdx.x * p.together * 2 * Sh::PART;
  int* meta = reinterpret_cast<int*>(reinterpret_cast<float*>(a.ws) + (long long)gridDim.x * p.together * 2 * Sh::PART) + 4 * blockIdx.x;
  int goes_on = 0;   // blocks behind this one that its last group goes on in, if it began here
  // (units take turns where there are more warps than queries: the nth is of warps `turn` = n mod `turns`)
  const int items = p.together * queries, turns = max(1, WARPS / items), turn = warp / items;
  for (int item = turns > 1 ? warp - turn * items : warp; item < items && turn < turns * (turns > 1 ? 1 : WARPS); item += turns > 1 ? items : WARPS) {
    const int place = item / queries, q = item - place * queries;
    int nth = 0;
    auto of_warp = [&](int r) { return (r >> 1) * p.together + place; };
    auto part = [&](int r) {
      return r & 1 ? reinterpret_cast<const float*>(smem + of_warp(r) * Sh::RING)
                   : reinterpret_cast<const float*>(smem + WARPS * Sh::RING) + of_warp(r) * Sh::PART;
    };
    const int2 of = lane < n_parts ? part_of[2 * of_warp(lane) + (lane & 1)] : make_int2(-1, 0);
    for (unsigned left = __ballot_sync(0xffffffffu, of.x >= 0); left;) {
      const int r0 = __ffs(left) - 1;
      const int b = __shfl_sync(0xffffffffu, of.x, r0), unit = __shfl_sync(0xffffffffu, of.y, r0) >> 1;
      const bool mine = of.x == b && of.y >> 1 == unit;
      const unsigned all = __ballot_sync(0xffffffffu, mine);
      left &= ~all;
      const bool here = r0 & 1, ends = __ballot_sync(0xffffffffu, mine && (of.y & 1));
      if (warp == 0 && item == 0 && here && !ends && !p.whole) {
        // the block that has the group's last step: the last k with total * k / blocks < the steps up to it
        goes_on = (int)(quot(part_upto[of_warp(r0)] * blocks + total - 1, max(1ll, total)) - 1 - blockIdx.x);
        if (lane == 0) meta[0] = b, meta[1] = unit;
      }
      const int head = p.tiles_by.of(unit), qi = (unit - head * p.tiles) * Sh::NQ + q;
      if (qi >= p.group || (turns > 1 && nth++ % turns != turn)) continue;
      const float4 v = mine ? *reinterpret_cast<const float4*>(part(lane) + Sh::NQ * DP + 4 * q) : make_float4(NONE, 0.f, 0.f, 0.f);
      float m = v.x;
#pragma unroll
      for (int k = 16; k; k >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
      const float less = ex2(v.x - m);
      float l = v.y * less, w = v.z * less;
#pragma unroll
      for (int k = 16; k; k >>= 1) {
        l += __shfl_xor_sync(0xffffffffu, l, k);
        w = fmaxf(w, __shfl_xor_sync(0xffffffffu, w, k));
      }
      const float by = less * moved(top_exp(v.z), top_exp(w));
      const int qh = head * p.group + qi;
      T* out = reinterpret_cast<T*>(a.out) + b * a.ldo + (long long)qh * dim;
      float* to = ws + (2 * place + here) * Sh::PART;
      const bool done = here && ends;
      const float f = done ? closing(l, w) : 1.f;
      for (int d = 4 * lane; d - 4 * lane < DP; d += 128) {
        const bool in = d < DP;
        float4 sum = make_float4(0, 0, 0, 0);
#pragma unroll 4
        for (unsigned rest = all; rest; rest &= rest - 1) {
          const int r = __ffs(rest) - 1;
          const float f = __shfl_sync(0xffffffffu, by, r);
          const float4 x = in ? *reinterpret_cast<const float4*>(part(r) + q * DP + d) : make_float4(0, 0, 0, 0);
          sum = make_float4(fmaf(x.x, f, sum.x), fmaf(x.y, f, sum.y), fmaf(x.z, f, sum.z), fmaf(x.w, f, sum.w));
        }
        if (!in) continue;
        if (done) {
          store_row(out, p.pairs, d, dim, sum.x * f, sum.y * f);
          store_row(out, p.pairs, d + 2, dim, sum.z * f, sum.w * f);
        } else if (!p.whole) {   // (whole units are done, unless lengths changed meanwhile: they may have no workspace)
          *reinterpret_cast<float4*>(to + q * DP + d) = sum;
        }
      }
      if (lane == 0) {
        if (done && a.lse) a.lse[(long long)b * a.q_heads + qh] = lse_of(m, l);
        if (!done && !p.whole) *reinterpret_cast<float4*>(to + Sh::NQ * DP + 4 * q) = make_float4(m, l, w, 0.f);
      }
    }
  }
  // (within the grid also where lengths changed meanwhile)
  if (!p.whole && threadIdx.x == 0) meta[2] = max(0, min(goes_on, (int)(gridDim.x - 1 - blockIdx.x)));
}

// Units of several blocks: block (x, y) joins some queries of a unit of the y-th group that goes over
// several blocks (no more than there are groups), over the parts in the line's order: their maxima and
// factors first, then a thread has four columns of a query over every `lanes`-th part.  Bound by the
// latency of its loads in turn: 2 us behind 1 x 131072 tokens of 16 + 4 heads (2.5 MB of parts).
//
// FEW: every block has an SM to itself.  Then a thread's first AHEAD parts are under way while the factors are
// found (107 registers): 1 x 131072 tokens 32.7 us, 35.3 without.  Else three blocks share one: 64 ragged sequences
// of 32 + 8 heads 104 us with, 99 without.
constexpr int JOIN = 512;
template <class T, int DP, int NT, bool FEW>
__global__ void __launch_bounds__(JOIN, FEW ? 1 : 3) k_kv_join(const __grid_constant__ KvCache c, const __grid_constant__ KvAttnArgs a,
                                                  const __grid_constant__ Plan p) {
  typedef Shape<T, DP, NT> Sh;
  __shared__ float by[Sh::NQ][GRID_MAX], stat[Sh::NQ][3];   // factors; m, l, w
  __shared__ float4 sums[JOIN];
  const int chunks = (min(Sh::NQ, p.group) + p.join_queries - 1) / p.join_queries;
  const int place = blockIdx.x / chunks, q0 = (blockIdx.x - place * chunks) * p.join_queries;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_trigger();
  pdl_wait();
  const float* ws = reinterpret_cast<const float*>(a.ws);
  const int4* metas = reinterpret_cast<const int4*>(ws + (long long)p.grid * p.together * 2 * Sh::PART);
  // the block that began it: the y-th one that says so
  int opens[GRID_MAX / 32], i = -1;
  int2 units[FEW ? GRID_MAX / 32 : 1], meta = make_int2(0, 0);
#pragma unroll
  for (int e = 0; e < GRID_MAX / 32; ++e) {
    const int4 v = FEW && lane + 32 * e < p.grid ? metas[lane + 32 * e] : make_int4(0, 0, 0, 0);
    opens[e] = FEW ? v.z : lane + 32 * e < p.grid ? metas[lane + 32 * e].z : 0;
    if (FEW) units[FEW ? e : 0] = make_int2(v.x, v.y);
  }
  int left = blockIdx.y, over = 0;   // blocks that it goes on in
#pragma unroll
  for (int e = 0; e < GRID_MAX / 32; ++e) {
    unsigned some = __ballot_sync(0xffffffffu, opens[e] > 0);
    const int n = __popc(some);
    if (i < 0 && left < n) {
      for (; left; --left) some &= some - 1;
      const int at = __ffs(some) - 1;
      i = 32 * e + at;
      over = __shfl_sync(0xffffffffu, opens[e], at);
      if (FEW) {
        const int2 v = units[FEW ? e : 0];
        meta = make_int2(__shfl_sync(0xffffffffu, v.x, at), __shfl_sync(0xffffffffu, v.y, at));
      }
    }
    left -= n;
  }
  if (i < 0) return;
  if (!FEW) meta = *reinterpret_cast<const int2*>(metas + i);
  const int n = min(over, p.grid - 1 - i) + 1;
  // (places of the tensors also where two calls share a workspace at the same time, which they must not)
  const int b = min((unsigned)meta.x, c.seqs - 1u), unit = min((unsigned)meta.y, (unsigned)(c.heads * p.tiles - p.together)) + place;
  const int head = p.tiles_by.of(unit), first = (unit - head * p.tiles) * Sh::NQ;
  const int queries = min(min(Sh::NQ, p.group - first) - q0, p.join_queries);
  if (queries <= 0) return;
  auto part = [&](int k) { return ws + (2ll * ((i + k) * p.together + place) + (k ? 0 : 1)) * Sh::PART; };
  constexpr int AHEAD = FEW ? 10 : 0;
  float4 ahead[AHEAD + 1];
  if constexpr (FEW) {
    const int width = queries * (DP / 4), lanes = JOIN / width, x = tid % width, k0 = tid / width;
    if (k0 < lanes)
#pragma unroll
      for (int e = 0; e < AHEAD; ++e)
        if (k0 + e * lanes < n) ahead[e] = *reinterpret_cast<const float4*>(part(k0 + e * lanes) + q0 * DP + 4 * x);
  }
  for (int q = warp; q < queries; q += JOIN / 32) {   // a warp to a query
    float4 v[GRID_MAX / 32];   // (all of them under way at once)
    float m = NONE, w = 0.f, l = 0.f;
#pragma unroll
    for (int e = 0; e < GRID_MAX / 32; ++e) {
      v[e] = make_float4(NONE, 0.f, 0.f, 0.f);
      if (lane + 32 * e < n) v[e] = *reinterpret_cast<const float4*>(part(lane + 32 * e) + Sh::NQ * DP + 4 * (q0 + q));
    }
#pragma unroll
    for (int e = 0; e < GRID_MAX / 32; ++e) m = fmaxf(m, v[e].x);
#pragma unroll
    for (int k = 16; k; k >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
#pragma unroll
    for (int e = 0; e < GRID_MAX / 32; ++e) {
      const float less = ex2(v[e].x - m);
      l += v[e].y * less;
      w = fmaxf(w, v[e].z * less);
      v[e].x = less;
    }
#pragma unroll
    for (int k = 16; k; k >>= 1) {
      l += __shfl_xor_sync(0xffffffffu, l, k);
      w = fmaxf(w, __shfl_xor_sync(0xffffffffu, w, k));
    }
#pragma unroll
    for (int e = 0; e < GRID_MAX / 32; ++e)
      if (lane + 32 * e < n) by[q][lane + 32 * e] = v[e].x * moved(top_exp(v[e].z), top_exp(w));
    if (lane == 0) stat[q][0] = m, stat[q][1] = l, stat[q][2] = w;
  }
  __syncthreads();
  const int width = queries * (DP / 4), lanes = JOIN / width, x = tid % width, k0 = tid / width;
  const int q = x / (DP / 4), d = 4 * (x - q * (DP / 4));
  float4 sum = make_float4(0, 0, 0, 0);
  if (k0 < lanes) {
    auto add = [&](const float4& v, int k) {
      const float w = by[q][k];
      sum = make_float4(fmaf(v.x, w, sum.x), fmaf(v.y, w, sum.y), fmaf(v.z, w, sum.z), fmaf(v.w, w, sum.w));
    };
#pragma unroll
    for (int e = 0; e < AHEAD; ++e)
      if (k0 + e * lanes < n) add(ahead[e], k0 + e * lanes);
#pragma unroll 5
    for (int k = k0 + AHEAD * lanes; k < n; k += lanes) add(*reinterpret_cast<const float4*>(part(k) + q0 * DP + 4 * x), k);
    sums[tid] = sum;
  }
  __syncthreads();
  if (k0) return;
  for (int k = 1; k < lanes; ++k) {
    const float4 v = sums[k * width + x];
    sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
  }
  const int qh = head * p.group + first + q0 + q;
  T* out = reinterpret_cast<T*>(a.out) + b * a.ldo + (long long)qh * c.head_dim;
  const float f = closing(stat[q][1], stat[q][2]);
  store_row(out, p.pairs, d, c.head_dim, sum.x * f, sum.y * f);
  store_row(out, p.pairs, d + 2, c.head_dim, sum.z * f, sum.w * f);
  if (a.lse && d == 0) a.lse[(long long)b * a.q_heads + qh] = lse_of(stat[q][0], stat[q][1]);
}

int padded(int dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }
int eights(int dim, int group) { return group > 8 && dim <= 128 ? 2 : 1; }
long long steps_of(int dim, long long tokens) { return (tokens + (dim > 128 ? 15 : 31)) / (dim > 128 ? 16 : 32); }

// Units that go together: as many of a sequence's as divide them and use seven of eight warps.
int together(int units, int warps) {
  int n = std::min(units, warps);
  while (units % n || 8 * n * (warps / n) < 7 * warps) --n;
  return n;
}

// Strides of page and slot in the largest power of two that divides both; false where the last
// place's offset does not fit 32 bits in it.
bool units_of(const KvCache& c, const long long (&stride)[3], unsigned (&unit)[2], unsigned* bytes) {
  const long long st[2] = {c.pages > 1 ? stride[0] : 0, c.page_size > 1 ? stride[1] : 0};
  int shift = 4;
  while (shift < 30 && !((st[0] | st[1]) >> shift & 1) && (st[0] | st[1])) ++shift;
  *bytes = 1u << shift;
  const unsigned __int128 last = (unsigned __int128)(c.pages - 1) * (st[0] >> shift) + (unsigned __int128)(c.page_size - 1) * (st[1] >> shift);
  for (int i = 0; i < 2; ++i) unit[i] = (unsigned)(st[i] >> shift);
  return last <= 0xffffffffu;
}

template <class T, int DP, int NT> cudaError_t attend(const KvCache& c, const KvAttnArgs& a, cudaStream_t s) {
  typedef Shape<T, DP, NT> Sh;
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
  p.page.by(c.page_size);
  p.group = a.q_heads / c.heads;
  p.tiles = (p.group + Sh::NQ - 1) / Sh::NQ;
  p.tiles_by.by(p.tiles);
  const int es = sizeof(T);
  p.pairs = !((uintptr_t)a.out & (2 * es - 1)) && a.ldo % 2 == 0;
  p.vectors = !((uintptr_t)a.q & (4 * es - 1)) && a.ldq % 4 == 0;
  p.scale = a.scale * 1.4426950408889634f;
  if (!units_of(c, c.k_stride, p.k_unit, &p.k_bytes) || !units_of(c, c.v_stride, p.v_unit, &p.v_bytes)) return cudaErrorNotSupported;
  for (int i = 0; i < 2; ++i) {   // (strides of one page or slot say nothing)
    const bool one = (i ? c.page_size : c.pages) == 1;
    p.ks[i] = one ? 0 : (unsigned)c.k_scale_stride[i];
    p.vs[i] = one ? 0 : (unsigned)c.v_scale_stride[i];
  }
  long long tokens = (long long)c.table_pages * c.page_size;
  if (a.window) tokens = std::min(tokens, (long long)a.window);
  const long long units = (long long)c.seqs * c.heads * p.tiles, steps = steps_of(c.head_dim, tokens);
  const long long to_block = (units + n_sms - 1) / n_sms;   // units, where every SM takes the same number of whole ones
  p.whole = !whole_units(units, steps, Sh::WARPS) ? 0 : to_block > Sh::WARPS ? 1 : 2;
  p.together = p.whole == 2 ? (int)to_block : p.whole ? 1 : together(c.heads * p.tiles, Sh::WARPS);
  p.split = Sh::WARPS / p.together;
  p.split_by.by(p.split);
  p.together_by.by(p.together);
  p.groups = c.heads * p.tiles / (p.whole == 2 ? 1 : p.together);
  p.units = p.whole == 2 ? (int)units : 0;
  p.groups_by.by(p.groups);
  // blocks: one to an SM; fewer where there are not two steps to a warp
  long long grid = std::min(n_sms, GRID_MAX);
  if (p.whole == 2) grid = (units + to_block - 1) / to_block;
  if (p.whole == 0) grid = std::min(grid, (units / p.together * steps + 2 * p.split - 1) / (2 * p.split));
  p.blocks_by.by((unsigned)grid);
  p.grid = (int)grid;
  // queries to a block of the second kernel: all of them where a unit has a few parts, fewer where
  // a few sequences have all blocks, so that at most four parts follow one another
  const int queries = std::min(Sh::NQ, p.group);
  const long long parts = grid / ((long long)c.seqs * p.groups);
  p.join_queries = queries;
  while (p.join_queries > 1 && 4 * (JOIN / (p.join_queries * (DP / 4))) < parts) --p.join_queries;
  e = launch_pdl(k_kv_attention<T, DP, NT>, (unsigned)grid, 32 * Sh::WARPS, Sh::SMEM, s, c, a, p);
  if (e != cudaSuccess) return e;
  e = launched();
  if (e != cudaSuccess || p.whole) return e;
  const dim3 joins(p.together * ((queries + p.join_queries - 1) / p.join_queries), (unsigned)std::min(grid, (long long)c.seqs * p.groups));
  e = joins.x * joins.y <= (unsigned)n_sms ? launch_pdl(k_kv_join<T, DP, NT, true>, joins, JOIN, 0, s, c, a, p)
                                           : launch_pdl(k_kv_join<T, DP, NT, false>, joins, JOIN, 0, s, c, a, p);
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
  const int group = q_heads / heads, queries = 8 * eights(dim, group), units = heads * ((group + queries - 1) / queries);
  // (by the fewest warps of a block of either type)
  if (whole_units((long long)seqs * units, steps_of(dim, tokens), queries > 8 || dim > 128 ? 8 : 12)) return 0;
  const size_t most = std::max({together(units, 8), together(units, 12), together(units, 16)});   // (by a block's warps)
  return GRID_MAX * (most * 2 * queries * (padded(dim) + 4) * 4 + 16);
}

cudaError_t launch_kv_attention(DType dt, const KvCache& c, const KvAttnArgs& a, cudaStream_t s) {
  return dt == F32 ? attend<float>(c, a, s) : attend<bf16>(c, a, s);
}

}  // namespace ff
