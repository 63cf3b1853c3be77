// 8-bit dense layers with a scale for each block of 128 (formula: featfix_op_gemm8),
// on the tensor cores (tcgen05.mma kind::f8f6f4, fp32 accumulators in TMEM).
//
// The scales change every 128 columns of K, so TMEM only ever holds the sum over one
// such block: the MMA warp fills an accumulator buffer with four K = 32 products and
// starts the next buffer, while the epilogue warps read the buffer back, multiply it
// by its two scales and add it to fp32 sums in their registers.  A row of a thread
// covers 128 columns, one scale block of W and of an 8-bit result, so a thread needs
// a single product of scales per block and finds the largest magnitude of an 8-bit
// result's block by itself.
#include "ff_common.cuh"
#include "ff_host.h"
#include "ff_q8.cuh"
#include "ff_tc.cuh"

#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <mutex>
#include <type_traits>

namespace ff {

namespace {

using namespace tc;

__device__ unsigned int g_watchdog8;

constexpr int BK = 128;   // one scale block, one 128-byte swizzled row of a stage

// Bounded wait: polls, and looks at the clock and the abort flag once in 256 polls
// only (reading the global timer takes long).  Written out at each use: a call would
// spill the epilogue's sums.
__device__ __forceinline__ bool wait_poll(uint64_t* b, uint32_t parity, volatile int* abort_flag,
                                          unsigned long long limit_ns = WAIT_LIMIT_NS) {
  unsigned long long t0 = 0;
#pragma unroll 1
  for (uint32_t i = 1;; ++i) {
    if (mbar_test(b, parity)) return true;
    if ((i & 255) == 0) {
      if (i == 256) t0 = gtimer();
      if (*abort_flag || gtimer() - t0 > limit_ns) {
        *abort_flag = 1;
        atomicOr(&g_watchdog8, 1u);
        return false;
      }
    }
  }
}
// every lane waits, the vote keeps the code around it warp-uniform
__device__ __forceinline__ bool wait_warp(uint64_t* b, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(0xffffffffu, wait_poll(b, parity, abort_flag));
}
// The hand-overs of TMEM, on which every block of K waits twice: try_wait suspends the
// warp between looks, so its polls are not in the way of the other warps', and the loop
// is as short as it gets, for the code around it competes for the instruction cache.
// A look that finds nothing lasts 4 us here (200 in a row 0.80 ms), however long it may be
// suspended for, so a million are the same 4 s; the watchdog's probe measures it.  (8192 x
// 8192 x 8192: 520 us with the polls above, 494 with this.)
constexpr int WAIT_LOOKS = 1000000;
template <int LOOKS = WAIT_LOOKS>
__device__ __forceinline__ bool wait_try(uint64_t* b, uint32_t parity, volatile int* abort_flag) {
  uint32_t n;
  asm volatile(
      "{\n .reg .pred p, q;\n .reg .u32 n;\n mov.u32 n, %4;\n"
      "LOOP_%=:\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n @p bra DONE_%=;\n"
      " sub.u32 n, n, 1;\n setp.ne.u32 q, n, 0;\n @q bra LOOP_%=;\n"
      "DONE_%=:\n mov.u32 %0, n;\n}\n"
      : "=r"(n)
      : "r"(saddr(b)), "r"(parity), "r"(100000u), "n"(LOOKS)
      : "memory");
  if (!__any_sync(0xffffffffu, n == 0)) return true;
  *abort_flag = 1;
  atomicOr(&g_watchdog8, 1u);
  return false;
}

// instruction descriptor, kind::f8f6f4: D fp32 (bit 4), A and B e4m3 (0 at bits 7
// and 10), both K-major, N >> 3 at bit 17, M >> 4 at bit 24
constexpr uint32_t idesc8(int m, int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24); }

__device__ __forceinline__ void umma8_pair(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(
          d_tmem),
      "l"(a), "l"(b), "r"(idesc), "r"(accum));
}

// 64 consecutive TMEM columns of this warp's lanes, read when it returns
__device__ __forceinline__ void tmem_ld64(uint32_t taddr, uint32_t (&r)[64]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32, %33, %34, %35, %36, %37, "
      "%38, %39, %40, %41, %42, %43, %44, %45, %46, %47, %48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, "
      "%60, %61, %62, %63}, [%64];\n"
      "tcgen05.wait::ld.sync.aligned;\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]), "=r"(r[32]),
        "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]), "=r"(r[40]),
        "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]), "=r"(r[48]),
        "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]), "=r"(r[56]),
        "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
      : "r"(taddr)
      : "memory");
}

// Arrival on an mbarrier of either CTA of a pair that only says that TMEM has been
// read (tcgen05.wait::ld and the tcgen05 fence are behind it): nothing in memory is
// handed over, so it is relaxed.  A release at cluster scope waited for the
// thread's stores every time: 8192 x 8192 x 8192 1133 us with it, 595 without.
__device__ __forceinline__ void arrive_read(uint32_t bar_cluster) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar_cluster) : "memory");
}

// GELU (tanh form) of four values: x (1 + tanh u) / 2 = x f, f = 1 / (1 + 2^t), t = -2 u
// log2(e).  One reciprocal for the four (16 a clock and SM against 32 for the
// exponential): each t is capped at 31, so that the four denominators' product stays
// finite.  A little more than the f of that cap is taken off, saturated to [0, 1], in
// the last product of f: it is exactly 0 from the cap on (x below -5.6), however
// large -x is, and minus infinity gives NaN as the formula does.  Within 2^-21 |x| and
// 3e-9 of the exact value; the hardware tanh (2^-11) would show in an 8-bit result's
// scales.
__device__ __forceinline__ void gelu4(f32x2& a, f32x2& b) {
  constexpr float C0 = -2.0f * 0.7978845608028654f * 1.4426950408889634f, C1 = C0 * 0.044715f;
  constexpr float CAP = 31.f, OFF = 0x1p-31f * (1.f + 0x1p-18f);
  const f32x2 k0 = f2u(C0, C0), k1 = f2u(C1, C1), one = f2u(1.f, 1.f);
  auto denominators = [&](f32x2 v) {
    const f32x2 t = fmul2(v, ffma2(fmul2(v, v), k1, k0));
    float e0, e1;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(fminf(lo_f(t), CAP)));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(fminf(hi_f(t), CAP)));
    return fadd2(f2u(e0, e1), one);
  };
  auto factor = [](float x, float y) { return __saturatef(__fmaf_rn(x, y, -OFF)); };
  const f32x2 da = denominators(a), db = denominators(b);
  const float pa = lo_f(da) * hi_f(da), pb = lo_f(db) * hi_f(db);
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(pa * pb));
  const float ra = r * pb, rb = r * pa;   // 1 / pa, 1 / pb
  a = f2u(lo_f(a) * factor(ra, hi_f(da)), hi_f(a) * factor(ra, lo_f(da)));
  b = f2u(lo_f(b) * factor(rb, hi_f(db)), hi_f(b) * factor(rb, lo_f(db)));
}

// ---------------------------------------------------------------------------
// CTA pairs: 256 x 256 tiles of the result, persistent.  Each CTA stages its own
// 128 rows of A and 128 of the tile's rows of W (32 KB a block of K) and
// holds 128 x 256 of the accumulator.
//   warp 0     TMA producer, a ring of STAGES blocks of K
//   warp 1     MMA issuer (even CTA): tcgen05.mma.cta_group::2, M = N = 256
//   warps 4-11 epilogue: TMEM lane quarter warp % 4, column half (warp - 4) / 4
// 168 registers a thread at launch; the first four warps hand theirs on down to
// 40, the epilogue's two warpgroups take 232 (40 + 2 * 232 = 3 * 168), 128 of
// which hold sums.  A spill in any role's loop costs more than anything else here
// (80 bytes: 8192 x 8192 x 8192 447 -> 718 us).
// Bound by the hand-over of the two TMEM buffers: a block of K takes about 820 clocks,
// 512 of them products; then by a tile's results, during which the products stand
// still but for two blocks.  Measured: 8192 x 8192 x 8192 430-460 us (2.4-2.6 PFLOP/s, at
// the power cap), 14310 x 2048 x 8192 with gate and residual 205-213 us (2.3), 14310 x
// 8192 x 2048 with GELU and 8-bit output 245-250 us (1.9).
// ---------------------------------------------------------------------------
constexpr int P_THREADS = 384;
constexpr int P_STAGES = 4;
constexpr uint32_t P_STAGE_BYTES = 2 * 128 * BK;
constexpr uint32_t P_EPI_BYTES = 8 * 8192;   // 8 KB of output blocks to an epilogue warp
constexpr uint32_t P_CONST_BYTES = 3 * 128 * 4;   // a warp's columns: bias, gate of its first and last row
constexpr size_t P_SMEM = 1024 + (size_t)P_STAGES * P_STAGE_BYTES + P_EPI_BYTES + 8 * P_CONST_BYTES + 256;

// 128-byte-swizzled block of 32 rows: 16-byte chunk k of row r
__device__ __forceinline__ uint32_t sw128_off(int r, int k) { return (uint32_t)(r * 128 + ((k ^ (r & 7)) << 4)); }

enum { STAGED = 1, RESID_TMA = 2 };

// Bias and gate of a warp's 128 columns, on their way into shared memory (cp.async)
// while the sums are formed, not read behind the last product (4096 x 1152 x 4608 with
// gate and residual 53.5 -> 48.4 us).
template <class T>
__device__ __forceinline__ void consts_in(const Gemm8Args& g, uint8_t* cst, int row0, int n0, int M, int N, int lane) {
  if (g.bias) {
    const T* bias = reinterpret_cast<const T*>(g.bias) + n0;
    if (!((uintptr_t)bias & 3)) {
      constexpr int E = 4 / (int)sizeof(T);
      for (int i = lane; i < 128 / E; i += 32)
        cp_async4(cst + 4 * i, n0 + E * i < N ? bias + E * i : bias, max(0, min(4, (N - n0 - E * i) * (int)sizeof(T))));
    } else {
      for (int i = lane; i < 128; i += 32) reinterpret_cast<T*>(cst)[i] = n0 + i < N ? bias[i] : from_f<T>(0.f);
    }
  }
  if (g.gate) {
    const float* lo = g.gate + (long long)(row0 / g.rpb) * g.gate_stride + n0;
    const float* hi = g.gate + (long long)(min(row0 + 31, M - 1) / g.rpb) * g.gate_stride + n0;
    for (int i = lane; i < 128; i += 32) {
      const bool in = n0 + i < N;
      cp_async4(cst + 512 + 4 * i, in ? lo + i : lo, in ? 4 : 0);
      cp_async4(cst + 1024 + 4 * i, in ? hi + i : hi, in ? 4 : 0);
    }
  }
  cp_commit();
}

// 16 bytes in shared memory as fp32 pairs
__device__ __forceinline__ void pairs16(const float* p, f32x2 (&v)[2]) {
  const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(p);
  v[0] = q.x; v[1] = q.y;
}
__device__ __forceinline__ void pairs16(const bf16* p, f32x2 (&v)[4]) {
  const uint4 q = *reinterpret_cast<const uint4*>(p);
  v[0] = bf2u(q.x); v[1] = bf2u(q.y); v[2] = bf2u(q.z); v[3] = bf2u(q.w);
}

// bias, GELU and gate of a row's columns n0 + c .. n0 + c + 31.  `gate`: the row's 128
// columns in shared memory, or null where the warp's rows have more than two samples
// (fewer than 32 rows to one).
template <class T, bool Q8>
__device__ __forceinline__ void finish32(const Gemm8Args& g, const uint8_t* cst, const float* gate, int m, int n0, int c,
                                         int N, f32x2* y) {
  if (g.bias) {
    constexpr int P = 8 / (int)sizeof(T);   // pairs to 16 bytes
#pragma unroll
    for (int j = 0; j < 16; j += P) {
      f32x2 b[P];
      pairs16(reinterpret_cast<const T*>(cst) + c + 2 * j, b);
#pragma unroll
      for (int i = 0; i < P; ++i) y[j + i] = fadd2(y[j + i], b[i]);
    }
  }
  if (g.act) {
#pragma unroll
    for (int j = 0; j < 16; j += 2) gelu4(y[j], y[j + 1]);
  }
  if (!Q8 && g.gate) {   // (8-bit results have none)
    if (gate) {
#pragma unroll
      for (int j = 0; j < 16; j += 2) {
        f32x2 f[2];
        pairs16(gate + c + 2 * j, f);
        y[j] = fmul2(y[j], f[0]);
        y[j + 1] = fmul2(y[j + 1], f[1]);
      }
    } else {
      const float* gp = g.gate + (long long)(m / g.rpb) * g.gate_stride + n0 + c;
#pragma unroll
      for (int j = 0; j < 16; ++j)
        y[j] = fmul2(y[j], f2u(n0 + c + 2 * j < N ? gp[2 * j] : 0.f, n0 + c + 2 * j + 1 < N ? gp[2 * j + 1] : 0.f));
    }
  }
}

// A warp's block of 32 rows of 128 bytes between shared memory and row-major global
// memory, for rows that TMA cannot take: four bytes to a lane where rows start on
// four, element by element otherwise.  block_in copies by cp.async where it can; its
// caller waits.  (Calls: written out, they would cost the loops their registers.)
template <class T>
__device__ __noinline__ void block_in(uint8_t* b, const T* src, long long ld, int rows, int cols, int lane) {
  constexpr int E = 4 / (int)sizeof(T);
  rows = min(rows, 32);
  if (!(((uintptr_t)src | (uintptr_t)(ld * sizeof(T))) & 3)) {
    const int bytes = max(0, min(4, (cols - E * lane) * (int)sizeof(T)));
    const T* p = bytes ? src + E * lane : src;
#pragma unroll 4
    for (int r = 0; r < rows; ++r, p += ld) cp_async4(b + sw128_off(r, lane >> 2) + (lane & 3) * 4, p, bytes);
  } else {
    // eight rows' loads in front of their stores (a load may not pass a store that could
    // alias it: 4000 x 2047 x 512 with a residual took 103 us row by row)
    for (int r0 = 0; r0 < rows; r0 += 8) {
      T v[8][E];
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e)
          v[i][e] = r0 + i < rows && lane + 32 * e < cols ? src[(r0 + i) * ld + lane + 32 * e] : from_f<T>(0.f);
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int j = lane + 32 * e;
          *reinterpret_cast<T*>(b + sw128_off(r0 + i, j * (int)sizeof(T) / 16) + j * sizeof(T) % 16) = v[i][e];
        }
    }
  }
}
template <class T>
__device__ __noinline__ void block_out(const uint8_t* b, T* dst, long long ld, int rows, int cols, int lane) {
  constexpr int E = 4 / (int)sizeof(T);
  rows = min(rows, 32);
  if (!(((uintptr_t)dst | (uintptr_t)(ld * sizeof(T))) & 3)) {
    const int n = cols - E * lane;   // elements of this lane's four bytes
    T* p = dst + E * lane;
    for (int r0 = 0; r0 < rows; r0 += 8) {   // (as in block_in: loads in front of stores)
      uint32_t v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const uint32_t*>(b + sw128_off(r0 + i, lane >> 2) + (lane & 3) * 4);
#pragma unroll
      for (int i = 0; i < 8; ++i, p += ld) {
        if (r0 + i >= rows) break;
        if (n >= E) {
          *reinterpret_cast<uint32_t*>(p) = v[i];
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (e < n) p[e] = reinterpret_cast<const T*>(&v[i])[e];
        }
      }
    }
  } else {
    for (int r0 = 0; r0 < rows; r0 += 8) {
      T v[8][E];
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int j = lane + 32 * e;
          v[i][e] = *reinterpret_cast<const T*>(b + sw128_off(r0 + i, j * (int)sizeof(T) / 16) + j * sizeof(T) % 16);
        }
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (r0 + i < rows && lane + 32 * e < cols) dst[(r0 + i) * ld + lane + 32 * e] = v[i][e];
    }
  }
}

// Sums of a thread's row over 128 columns -> result, through the warp's two 4 KB
// blocks.  A TMA store writes whole 16 bytes, past the last column too: rows that
// do not end on 16 bytes leave their last tile through block_out.
template <class T, bool Q8>
__device__ __forceinline__ bool finish_row(const Gemm8Args& g, int flags, const CUtensorMap* tmO, f32x2 (&acc)[64], int row0,
                                           int lane, int n0, int M, int N, uint8_t* blk, const uint8_t* cst, uint64_t* rbar,
                                           uint32_t rph, volatile int* abort_flag) {
  cp_wait<0>();
  __syncwarp();
  const int m = min(row0 + lane, M - 1);   // (rows past M repeat the last one and are not stored)
  const int es = Q8 ? 1 : (int)sizeof(T);
  const float* gate = nullptr;
  if (!Q8 && g.gate) {
    const int b_lo = row0 / g.rpb, b_hi = min(row0 + 31, M - 1) / g.rpb;
    if (b_hi - b_lo <= 1) gate = reinterpret_cast<const float*>(cst + (m / g.rpb == b_lo ? 512 : 1024));
  }
  const bool tma = (flags & STAGED) && (n0 + 128 <= N || (long long)N * es % 16 == 0);
  if constexpr (Q8) {
    // (columns past N are sums over rows of zeros: GELU and magnitude 0)
    float mx = 0.f;
#pragma unroll
    for (int c = 0; c < 128; c += 32) {
      finish32<T, Q8>(g, cst, gate, m, n0, c, N, acc + c / 2);
#pragma unroll
      for (int j = c / 2; j < c / 2 + 16; ++j) {
        mx = max_abs(mx, max_abs(lo_f(acc[j]), hi_f(acc[j])));
      }
    }
    const float s = q8_scale(__float_as_uint(mx)), inv = q8_inv(s);
    if (row0 + lane < M) g.q8.scale[(n0 >> 7) * g.q8.lds + m] = s;
    if (lane == 0) bulk_wait_read<0>();
    __syncwarp();
    const f32x2 i2 = f2u(inv, inv);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x2 u = fmul2(acc[8 * k + 2 * i], i2), v = fmul2(acc[8 * k + 2 * i + 1], i2);
        w[i] = to_e4m3x4(lo_f(u), hi_f(u), lo_f(v), hi_f(v));
      }
      *reinterpret_cast<uint4*>(blk + sw128_off(lane, k)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (tma) fence_async_smem();
    __syncwarp();
    if (!tma) {
      block_out<uint8_t>(blk, reinterpret_cast<uint8_t*>(g.q8.q) + row0 * g.q8.ldq + n0, g.q8.ldq, M - row0, N - n0, lane);
      __syncwarp();
    } else if (lane == 0) {
      tma_store(tmO, blk, n0, row0);
      bulk_commit();
    }
    return true;
  }
  constexpr int PER = 128 / (int)sizeof(T);   // columns of a block
  constexpr int V = 16 / (int)sizeof(T);
  if ((flags & RESID_TMA) && !wait_warp(rbar, rph, abort_flag)) return false;
#pragma unroll
  for (int c = 0; c < 128; c += PER) {
    if (n0 + c >= N) break;
    uint8_t* b = blk + (c / PER & 1) * 4096;
    if (!g.resid || c >= 2 * PER) {
      // the last tile's stores, or this tile's before last, have left the block (where
      // the residual is in it: before that came)
      if (lane == 0) {
        if (c == 0) bulk_wait_read<0>(); else bulk_wait_read<1>();
      }
      __syncwarp();
      if (g.resid) {   // (fp32: the third and fourth block)
        block_in<T>(b, reinterpret_cast<const T*>(g.resid) + row0 * g.ldr + n0 + c, g.ldr, M - row0, N - n0 - c, lane);
        cp_commit();
        cp_wait<0>();
        __syncwarp();
      }
    }
#pragma unroll
    for (int d = 0; d < PER; d += 32) {
      f32x2* y = acc + (c + d) / 2;
      finish32<T, Q8>(g, cst, gate, m, n0, c + d, N, y);
#pragma unroll
      for (int k = 0; k < 32 / V; ++k) {
        T* p = reinterpret_cast<T*>(b + sw128_off(lane, d / V + k));
        f32x2* u = y + V / 2 * k;
        if (g.resid) {
          f32x2 r[V / 2];
          pairs16(p, r);
#pragma unroll
          for (int i = 0; i < V / 2; ++i) u[i] = fadd2(u[i], r[i]);
        }
        float o[V];
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
          o[2 * i] = lo_f(u[i]);
          o[2 * i + 1] = hi_f(u[i]);
        }
        st16(p, o);
      }
    }
    if (tma) fence_async_smem();
    __syncwarp();
    if (!tma) {
      block_out<T>(b, reinterpret_cast<T*>(g.out) + row0 * g.ldo + n0 + c, g.ldo, M - row0, N - n0 - c, lane);
      __syncwarp();
    } else if (lane == 0) {
      tma_store(tmO, b, n0 + c, row0);
      bulk_commit();
    }
  }
  return true;
}

// Tile order: groups of 8 row blocks, each swept over all column blocks with its
// rows fastest (ff_gemm_tc.cu has the measurement).
__device__ __forceinline__ void tile_at8(int tile, int num_m, int num_n, int& m, int& n) {
  const int g = tile / (8 * num_n), r = tile - g * 8 * num_n;
  const int gm = min(8, num_m - g * 8);
  n = r / gm;
  m = g * 8 + r - n * gm;
}

template <class T, bool Q8>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(P_THREADS, 1)
    k_gemm8_pair(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmW,
                 const __grid_constant__ CUtensorMap tmO, const __grid_constant__ CUtensorMap tmR, int M, int N, int K,
                 int flags, const __grid_constant__ Gemm8Args g) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* epi = smem + P_STAGES * P_STAGE_BYTES;
  uint64_t* full = reinterpret_cast<uint64_t*>(epi + P_EPI_BYTES + 8 * P_CONST_BYTES);
  uint64_t* empty = full + P_STAGES;
  uint64_t* tfull = empty + P_STAGES;
  uint64_t* tempty = tfull + 2;
  uint64_t* rbar = tempty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(rbar + 8);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
  const int num_m = (M + 255) / 256, num_n = (N + 255) / 256, num_tiles = num_m * num_n;
  const int num_kb = (K + BK - 1) / BK;

  if (threadIdx.x == 0) {
    for (int s = 0; s < P_STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&tfull[b], 1);
      mbar_init(&tempty[b], 16);   // the epilogue warps of both CTAs
    }
    for (int w = 0; w < 8; ++w) mbar_init(&rbar[w], 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)&tmA) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)&tmW) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(saddr(tmem_slot)), "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncwarp();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_trigger();
  pdl_wait();

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp == 0 && lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (int tile = pair; tile < num_tiles && ok; tile += npairs) {
        int mb, nb;
        tile_at8(tile, num_m, num_n, mb, nb);
        for (int kb = 0; kb < num_kb; ++kb, ++it) {
          const int s = it % P_STAGES;
          if (!wait_poll(&empty[s], ((it / P_STAGES) & 1) ^ 1, abort_flag)) { ok = false; break; }
          if (rank == 0) mbar_expect_tx(&full[s], 2 * P_STAGE_BYTES);
          const uint32_t fb = map_to(&full[s], 0);
          uint8_t* st = smem + s * P_STAGE_BYTES;
          tma_load_pair(&tmA, fb, st, kb * BK, mb * 256 + (int)rank * 128);
          tma_load_pair(&tmW, fb, st + 128 * BK, kb * BK, nb * 256 + (int)rank * 128);
        }
      }
      if (rank == 0) {   // no copy may land after the CTAs exit
        for (uint32_t k = 0; k < (uint32_t)P_STAGES && k < it; ++k) {
          const uint32_t j = it - 1 - k;
          const unsigned long long t0 = gtimer();
          while (!mbar_try(&full[j % P_STAGES], (j / P_STAGES) & 1))
            if (gtimer() - t0 > WAIT_LIMIT_NS) { atomicOr(&g_watchdog8, 2u); break; }
        }
      }
    }
    if (warp == 1 && rank == 0) {
      const bool mine = elect_one();   // (here: every instruction between a free buffer and its products counts)
      uint32_t it = 0;   // blocks of K over all tiles: ring stage it % STAGES, TMEM buffer it % 2
      bool ok = true;
      for (int tile = pair; tile < num_tiles && ok; tile += npairs) {
        for (int kb = 0; kb < num_kb; ++kb, ++it) {
          const int s = it % P_STAGES;
          const uint32_t buf = it & 1;
          // the buffer comes last: it is what the next products wait for
          const uint32_t st = saddr(smem + s * P_STAGE_BYTES);
          const uint64_t ad = sw128_desc(st), wd = sw128_desc(st + 128 * BK);
          if (!wait_warp(&full[s], (it / P_STAGES) & 1, abort_flag) ||
              !wait_try(&tempty[buf], ((it >> 1) & 1) ^ 1, abort_flag)) { ok = false; break; }
          tc_fence_after();
          if (mine) {
#pragma unroll
            for (int k = 0; k < 4; ++k)   // 32 bytes along K inside the swizzle atom
              umma8_pair(tmem_base + buf * 256, ad + 2 * k, wd + 2 * k, idesc8(256, 256), k != 0);
            umma_commit_pair(&tfull[buf]);
            umma_commit_pair(&empty[s]);
          }
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
    const int q = warp & 3, h = (warp - 4) >> 2;
    uint8_t* blk = epi + (warp - 4) * 8192;
    uint8_t* cst = epi + P_EPI_BYTES + (warp - 4) * P_CONST_BYTES;
    const uint32_t tq = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(h * 128);
    const uint32_t tempty0 = map_to(tempty, 0);
    uint32_t it = 0, rph = 0;
    // a warp's first row and column of a tile; whether any of it is in the result
    auto place = [&](int tile, int& row0, int& n0) {
      int mb, nb;
      tile_at8(tile, num_m, num_n, mb, nb);
      row0 = mb * 256 + (int)rank * 128 + q * 32;
      n0 = nb * 256 + h * 128;
      return n0 < N && row0 < M;
    };
    // Scales of this row and of W's block of rows, two blocks of K ahead; a tile's first
    // ones are loaded in front of the tile before's results
    float a0 = 0.f, w0 = 0.f, a1 = 0.f, w1 = 0.f;
    auto first_scales = [&](int tile) {
      int row0, n0;
      if (tile >= num_tiles || !place(tile, row0, n0) || row0 + lane >= M) return;
      const float* sa = g.sa + row0 + lane;
      const float* sw = g.sw + (n0 >> 7) * g.ldsw;
      a0 = sa[0];
      w0 = sw[0];
      if (num_kb > 1) {
        a1 = sa[g.ldsa];
        w1 = sw[1];
      }
    };
    first_scales(pair);
    for (int tile = pair; tile < num_tiles; tile += npairs) {
      int row0, n0;
      const bool live = place(tile, row0, n0);   // (warp-uniform)
      // the residual's copies begin a block of K late: the last tile's stores have left by then
      const int rk = live && !Q8 && g.resid ? min(1, num_kb - 1) : -1;
      bool resid_on = false;
      if (live) {
        __syncwarp();   // the last tile's are read
        consts_in<T>(g, cst, row0, n0, M, N, lane);
      }
      const bool in = live && row0 + lane < M;
      const float* sa = g.sa + row0 + lane;
      const float* sw = g.sw + (n0 >> 7) * g.ldsw;
      f32x2 acc[64];
#pragma unroll
      for (int i = 0; i < 64; ++i) acc[i] = 0;
      bool ok = true;
      for (int kb = 0; kb < num_kb; ++kb, ++it) {
        const uint32_t buf = it & 1;
        const float f = a0 * w0;
        a0 = a1;
        w0 = w1;
        if (in && kb + 2 < num_kb) {
          a1 = sa[(kb + 2) * g.ldsa];
          w1 = sw[kb + 2];
        }
        if (kb == rk) {
          if (lane == 0) bulk_wait_read<0>();
          __syncwarp();
          if (flags & RESID_TMA) {
            resid_on = true;
            if (lane == 0) {
              fence_async_smem();    // (block_out's reads)
              mbar_expect_tx(&rbar[warp - 4], n0 + 64 < N ? 8192u : 4096u);
              tma_load(&tmR, &rbar[warp - 4], blk, n0, row0);
              if (n0 + 64 < N) tma_load(&tmR, &rbar[warp - 4], blk + 4096, n0 + 64, row0);
            }
          } else {
            constexpr int PER = 128 / (int)sizeof(T);
            const T* rp = reinterpret_cast<const T*>(g.resid) + row0 * g.ldr + n0;
            block_in<T>(blk, rp, g.ldr, M - row0, N - n0, lane);
            if (n0 + PER < N) block_in<T>(blk + 4096, rp + PER, g.ldr, M - row0, N - n0 - PER, lane);
            cp_commit();
          }
          __syncwarp();
        }
        if (!wait_try(&tfull[buf], (it >> 1) & 1, abort_flag)) { ok = false; break; }
        tc_fence_after();
        if (live) {
          const f32x2 ff = f2u(f, f);
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t p[64];
            tmem_ld64(tq + buf * 256 + c * 64, p);
            if (c == 1) {   // the buffer is read: the MMA warp may fill it again
              tc_fence_before();
              if (lane == 0) arrive_read(tempty0 + 8 * buf);
            }
#pragma unroll
            for (int i = 0; i < 32; ++i)
              acc[c * 32 + i] = ffma2((f32x2)p[2 * i] | (f32x2)p[2 * i + 1] << 32, ff, acc[c * 32 + i]);
          }
        } else {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_read(tempty0 + 8 * buf);
        }
      }
      first_scales(tile + npairs);
      if (ok && live) {
        ok = finish_row<T, Q8>(g, flags, &tmO, acc, row0, lane, n0, M, N, blk, cst, &rbar[warp - 4], rph, abort_flag);
      } else if (!ok && resid_on && lane == 0) {   // its copies still land before the CTA exits
        const unsigned long long t0 = gtimer();
        while (!mbar_try(&rbar[warp - 4], rph))
          if (gtimer() - t0 > WAIT_LIMIT_NS) { atomicOr(&g_watchdog8, 2u); break; }
      }
      if (live) rph ^= 1;
      if (!ok) break;
    }
    if (lane == 0) bulk_wait_all();
  }
  tc_fence_before();
  __syncwarp();
  cluster_sync_all();   // no CTA leaves while its peer may still address its TMEM or barriers
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512) : "memory");
  }
}

// ---------------------------------------------------------------------------
// Few rows of A: the product transposed.  128 rows of W are the M side of the
// products, BT rows of A (16 to 64) their N side, and the blocks of K are shared out
// to the S CTAs of a cluster, so that a handful of rows still reads W on every SM.
// A thread holds one row of W for BT / 2 rows of A; the scales' products are the same
// for all of them and come from shared memory.  The cluster's partial sums meet in
// shared memory: CTA r adds up and finishes the r-th share of the tile's rows of A, in
// the order of the CTAs (the same bits every time).
//   warp 0 TMA producer, warp 1 MMA issuer, warps 2-9 epilogue: TMEM lane quarter
//   warp % 4, half of the BT columns (warp - 2) / 4
// Bound by latencies in a row with few blocks of K (start, first copies, the cluster's
// meeting: 1 x 6144 x 2048 5.6 us, 1 x 2048 x 8192 6.8) and by the tiles' traffic from L2
// with many CTAs (256 x 2048 x 8192 16.6 us with a bias, 18.3 with gate and residual, 100
// MB of tiles).
// ---------------------------------------------------------------------------
constexpr int S_THREADS = 320;
constexpr int S_TABLE = 32;   // blocks of K whose scales are in shared memory at a time
template <int BT> struct SCfg {
  // two CTAs to an SM (deeper rings with one CTA were slower, clusters of
  // eight by half: 1 x 2048 x 8192 6.6 -> 12.4 us)
  static constexpr int STAGES = BT == 16 ? 5 : 4;
  static constexpr uint32_t STAGE_BYTES = (128 + BT) * BK;
  static constexpr uint32_t PART_BYTES = BT * 512;   // the tile in fp32
  // up to 32 rows the partial sums have a place of their own, above it they take the
  // ring's (with a cluster barrier more, until all are done with theirs)
  static constexpr bool OWN = BT <= 32;
  static constexpr size_t SMEM = 1024 + STAGES * STAGE_BYTES + (OWN ? PART_BYTES : 0) + S_TABLE * BT * 4 + 8 * BT * 4 + 256;
};

__device__ __forceinline__ void umma8(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(
          d_tmem),
      "l"(a), "l"(b), "r"(idesc), "r"(accum));
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n"
      "tcgen05.wait::ld.sync.aligned;\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
      : "r"(taddr)
      : "memory");
}
template <int C> __device__ __forceinline__ void tmem_read(uint32_t taddr, uint32_t (&r)[C]) {
  if constexpr (C == 8) tmem_ld8(taddr, r);
  else {
    float v[C];
    if constexpr (C == 32) tmem_ld32(taddr, v); else tmem_ld16(taddr, v);
#pragma unroll
    for (int i = 0; i < C; ++i) r[i] = __float_as_uint(v[i]);
  }
}
__device__ __forceinline__ void st_cluster(uint32_t addr, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void epi_barrier() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

template <class T, bool Q8, int BT>
__global__ void __launch_bounds__(S_THREADS, 2)
    k_gemm8_split(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmW, int M, int N, int K,
                  int S, const __grid_constant__ Gemm8Args g) {
  using C = SCfg<BT>;
  constexpr int CT = BT / 2;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  float* table = reinterpret_cast<float*>(smem + C::STAGES * C::STAGE_BYTES);   // [S_TABLE][BT]
  uint32_t* red = reinterpret_cast<uint32_t*>(table + S_TABLE * BT);             // [warp][row of A]
  uint64_t* full = reinterpret_cast<uint64_t*>(red + 8 * BT);
  uint64_t* empty = full + C::STAGES;
  uint64_t* tfull = empty + C::STAGES;
  uint64_t* tempty = tfull + 4;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tempty + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* part = C::OWN ? reinterpret_cast<float*>(tmem_slot + 4) : reinterpret_cast<float*>(smem);   // [S][BT / S][128]

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = S > 1 ? (int)cluster_rank() : 0;
  const int tile = blockIdx.x / S, num_a = (M + BT - 1) / BT;
  const int n0 = tile / num_a * 128, m0 = tile % num_a * BT;
  const int num_kb = (K + BK - 1) / BK;
  const int kb0 = (int)((long long)num_kb * rank / S), kb1 = (int)((long long)num_kb * (rank + 1) / S);

  if (threadIdx.x == 0) {
    for (int i = 0; i < C::STAGES; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int b = 0; b < 4; ++b) {
      mbar_init(&tfull[b], 1);
      mbar_init(&tempty[b], 8);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)&tmA) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)&tmW) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(saddr(tmem_slot)), "r"(4 * BT)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  if (C::OWN && S > 1) cluster_arrive();
  pdl_trigger();
  pdl_wait();

  const int q = warp & 3, h = (warp - 2) >> 2, row = q * 32 + lane;
  f32x2 acc[CT / 2];
#pragma unroll
  for (int i = 0; i < CT / 2; ++i) acc[i] = 0;
  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      for (int kb = kb0; kb < kb1; ++kb, ++it) {
        const int s = it % C::STAGES;
        if (!wait_poll(&empty[s], ((it / C::STAGES) & 1) ^ 1, abort_flag)) break;
        mbar_expect_tx(&full[s], C::STAGE_BYTES);
        uint8_t* st = smem + s * C::STAGE_BYTES;
        tma_load(&tmW, &full[s], st, kb * BK, n0);
        tma_load(&tmA, &full[s], st + 128 * BK, kb * BK, m0);
      }
      for (uint32_t k = 0; k < (uint32_t)C::STAGES && k < it; ++k) {   // no copy may land after the CTA exits
        const uint32_t j = it - 1 - k;
        const unsigned long long t0 = gtimer();
        while (!mbar_try(&full[j % C::STAGES], (j / C::STAGES) & 1))
          if (gtimer() - t0 > WAIT_LIMIT_NS) { atomicOr(&g_watchdog8, 2u); break; }
      }
    }
  } else if (warp == 1) {
    // the loop's time is this warp's: both barriers are tested together, and the next
    // block's behind this one's products
    const bool mine = elect_one();
    uint32_t it = 0;
    bool ready = false;
    for (int kb = kb0; kb < kb1; ++kb, ++it) {
      const int s = it % C::STAGES;
      const uint32_t buf = it & 3, st = saddr(smem + s * C::STAGE_BYTES);
      const uint64_t wd = sw128_desc(st), ad = sw128_desc(st + 128 * BK);
      if (!__all_sync(0xffffffffu, ready) && (!wait_warp(&tempty[buf], ((it >> 2) & 1) ^ 1, abort_flag) ||
                                              !wait_warp(&full[s], (it / C::STAGES) & 1, abort_flag)))
        break;
      tc_fence_after();
      {
        const uint32_t j = it + 1;
        const bool t = mbar_test(&tempty[j & 3], ((j >> 2) & 1) ^ 1), f = mbar_test(&full[j % C::STAGES], (j / C::STAGES) & 1);
        ready = t && f;
      }
      if (mine) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          umma8(tmem_base + buf * BT, wd + 2 * k, ad + 2 * k, idesc8(128, BT), k != 0);
        umma_commit(&tfull[buf]);
        umma_commit(&empty[s]);
      }
    }
  } else {
    const uint32_t tq = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(h * CT);
    const float* sw = g.sw + (n0 >> 7) * g.ldsw;
    uint32_t it = 0;
    bool ok = true, ready = false;   // (after a wait that gave up the loop still meets the others at its barriers)
    for (int kb = kb0; kb < kb1; ++kb, ++it) {
      if (it % S_TABLE == 0) {   // the scales' products of the next blocks of K
        if (it) epi_barrier();
        for (int i = threadIdx.x - 64; i < min(S_TABLE, kb1 - kb) * BT; i += 256) {
          const int b = kb + i / BT, m = m0 + i % BT;
          table[i] = m < M ? g.sa[b * g.ldsa + m] * sw[b] : 0.f;
        }
        epi_barrier();
      }
      const uint32_t buf = it & 3;
      if (!__all_sync(0xffffffffu, ready)) ok = ok && wait_warp(&tfull[buf], (it >> 2) & 1, abort_flag);
      if (!ok) continue;
      tc_fence_after();
      uint32_t p[CT];
      tmem_read<CT>(tq + buf * BT, p);
      tc_fence_before();
      if (lane == 0) mbar_arrive(&tempty[buf]);
      ready = mbar_test(&tfull[(it + 1) & 3], ((it + 1) >> 2) & 1);
      const float* f = table + it % S_TABLE * BT + h * CT;
#pragma unroll
      for (int i = 0; i < CT; i += 4) {
        const ulonglong2 f2 = *reinterpret_cast<const ulonglong2*>(f + i);
        acc[i / 2] = ffma2((f32x2)p[i] | (f32x2)p[i + 1] << 32, f2.x, acc[i / 2]);
        acc[i / 2 + 1] = ffma2((f32x2)p[i + 2] | (f32x2)p[i + 3] << 32, f2.y, acc[i / 2 + 1]);
      }
    }
  }
  // partial sums to the CTA that finishes their rows of A: part[CTA][row of A][row of W]
  const int lshare = (BT == 64 ? 6 : BT == 32 ? 5 : 4) - (31 - __clz(S)), share = 1 << lshare;
  __syncwarp();
  if (S == 1) {
    __syncthreads();
  } else {
    if (!C::OWN) cluster_arrive();   // (with OWN: every CTA of the cluster has started, above)
    cluster_wait();
  }
  if (warp >= 2) {
    const uint32_t at = saddr(part) + 4 * ((rank << lshare) * 128 + row);
#pragma unroll
    for (int i = 0; i < CT; ++i) {
      const int t = h * CT + i;
      const float v = i & 1 ? hi_f(acc[i / 2]) : lo_f(acc[i / 2]);
      const uint32_t to = at + (t & (share - 1)) * 512;
      if (S == 1) {
        part[t * 128 + row] = v;
      } else {
        uint32_t a;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(to), "r"(t >> lshare));
        st_cluster(a, v);
      }
    }
  }
  __syncwarp();
  if (S > 1) cluster_sync_all(); else __syncthreads();
  if (warp >= 2) {
    const int n = n0 + row, mine = share / 2, t0 = h * mine;   // this half's rows of A: t0 .. t0 + mine - 1 of the share
    const int mb = m0 + rank * share + t0, cnt = n < N ? min(mine, M - mb) : 0;
    const float bias = g.bias && n < N ? to_f(reinterpret_cast<const T*>(g.bias)[n]) : 0.f;
    float* const pp = part + t0 * 128 + row;
    constexpr int U = BT == 16 ? 4 : BT == 32 ? 8 : 16;   // rows of A at a time: their loads come first
    for (int u = 0; u < mine; u += U) {
      float y[U], gt[U], rs[U];
      if (!Q8) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const bool in = u + i < cnt;
          const long long m = mb + u + i;
          gt[i] = g.gate && in ? g.gate[(int)m / g.rpb * g.gate_stride + n] : 1.f;
          rs[i] = g.resid && in ? to_f(reinterpret_cast<const T*>(g.resid)[m * g.ldr + n]) : 0.f;
        }
      }
#pragma unroll
      for (int i = 0; i < U; ++i) y[i] = u + i < mine ? pp[(u + i) * 128] : 0.f;
      for (int s = 1; s < S; ++s) {
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (u + i < mine) y[i] += pp[(u + i) * 128 + (s << lshare) * 128];
      }
#pragma unroll
      for (int i = 0; i < U; ++i) y[i] += bias;
      if (g.act) {
#pragma unroll
        for (int i = 0; i < U; i += 4) {
          f32x2 p = f2u(y[i], y[i + 1]), r = f2u(y[i + 2], y[i + 3]);
          gelu4(p, r);
          y[i] = lo_f(p); y[i + 1] = hi_f(p); y[i + 2] = lo_f(r); y[i + 3] = hi_f(r);
        }
      }
      if constexpr (Q8) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
          if (u + i >= mine) break;
          const float v = n < N ? y[i] : 0.f;
          pp[(u + i) * 128] = v;
          const uint32_t mx = __reduce_max_sync(0xffffffffu, abs_bits(v));
          if (lane == 0) red[(t0 + u + i) * 4 + q] = mx;
        }
      } else {
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (u + i < cnt)
            reinterpret_cast<T*>(g.out)[(long long)(mb + u + i) * g.ldo + n] = from_f<T>(y[i] * gt[i] + rs[i]);
      }
    }
    if constexpr (Q8) {
      epi_barrier();
#pragma unroll 4
      for (int t = 0; t < cnt; ++t) {
        const uint4 r = *reinterpret_cast<const uint4*>(red + (t0 + t) * 4);
        const float sc = q8_scale(max(max(r.x, r.y), max(r.z, r.w)));
        reinterpret_cast<uint8_t*>(g.q8.q)[(mb + t) * g.q8.ldq + n] = (uint8_t)to_e4m3x2(pp[t * 128] * q8_inv(sc), 0.f);
        if (row == 0) g.q8.scale[(n0 >> 7) * g.q8.lds + mb + t] = sc;
      }
    }
  }
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(4 * BT) : "memory");
  }
}

// Both waits, on barriers that nothing arrives on, with a part of their limits: what they
// took, in ns.
constexpr int PROBE_PART = 32;
__device__ unsigned long long g_probe_ns[2];
__global__ void __launch_bounds__(64) k_gemm8_probe() {
  __shared__ uint64_t bar[2];
  __shared__ int abort_flag[2];
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bar[i], 1);
      abort_flag[i] = 0;
    }
  }
  __syncthreads();
  const int warp = threadIdx.x >> 5;
  const unsigned long long t0 = gtimer();
  if (warp == 0) wait_poll(&bar[0], 0, &abort_flag[0], WAIT_LIMIT_NS / PROBE_PART);
  else wait_try<WAIT_LOOKS / PROBE_PART>(&bar[1], 0, &abort_flag[1]);
  __syncwarp();
  if ((threadIdx.x & 31) == 0) g_probe_ns[warp] = gtimer() - t0;
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
PFN_cuTensorMapEncodeTiled_v12000 g_encode = nullptr;
std::once_flag g_once;

bool init_driver() {
  std::call_once(g_once, [] {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      g_encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
  });
  return g_encode != nullptr;
}

// SMs of the current device; its first call sets the kernels' shared-memory limits there
// (both are a device's own).
PerDevice<int> g_devices;
cudaError_t device_sms(int* sms) {
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= g_devices.devices) return cudaErrorInvalidDevice;
  return g_devices.get(dev, sms, [&](int& n) {
    cudaError_t first = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    auto smem = [&](const void* fn, size_t bytes) {
      const cudaError_t r = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
      if (first == cudaSuccess) first = r;
    };
    auto both = [&](auto t, auto q8) {
      using T = decltype(t);
      constexpr bool Q8 = decltype(q8)::value;
      smem((const void*)k_gemm8_pair<T, Q8>, P_SMEM);
      smem((const void*)k_gemm8_split<T, Q8, 16>, SCfg<16>::SMEM);
      smem((const void*)k_gemm8_split<T, Q8, 32>, SCfg<32>::SMEM);
      smem((const void*)k_gemm8_split<T, Q8, 64>, SCfg<64>::SMEM);
    };
    both(0.f, std::false_type());
    both(0.f, std::true_type());
    both(bf16(), std::false_type());
    both(bf16(), std::true_type());
    return first;
  });
}

// Row-major [rows, cols] of `es`-byte elements in boxes of box_rows rows of 128
// bytes, 128-byte swizzle, zero fill out of bounds.
bool make_map8(CUtensorMap* m, const void* base, int es, long long rows, long long cols, long long ld, int box_rows) {
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ld * es};
  cuuint32_t box[2] = {(cuuint32_t)(128 / es), (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1, 1};
  const CUtensorMapDataType t = es == 1   ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                                : es == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                          : CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
  return g_encode(m, t, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class T, bool Q8, int BT>
cudaError_t launch_split(int M, int N, int K, int S, const Gemm8Args& g, cudaStream_t s) {
  CUtensorMap ma, mw;
  if (!make_map8(&ma, g.a, 1, M, K, g.lda, BT) || !make_map8(&mw, g.w, 1, N, K, g.ldw, 128)) return cudaErrorInvalidValue;
  const long long grid = (long long)S * ((N + 127) / 128) * ((M + BT - 1) / BT);
  if (grid > 0x7fffffff) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(S_THREADS);
  cfg.dynamicSmemBytes = SCfg<BT>::SMEM;
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)S;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, k_gemm8_split<T, Q8, BT>, ma, mw, M, N, K, S, g);
  return e != cudaSuccess ? e : launched();
}

template <class T, bool Q8>
cudaError_t launch_pair(int M, int N, int K, int sms, const Gemm8Args& g, cudaStream_t s) {
  constexpr int es = (int)sizeof(T);
  CUtensorMap ma, mw, mo, mr;
  if (!make_map8(&ma, g.a, 1, M, K, g.lda, 128) || !make_map8(&mw, g.w, 1, N, K, g.ldw, 128))
    return cudaErrorInvalidValue;
  mo = mr = ma;
  int flags = 0;
  if (Q8) {
    if (!make_map8(&mo, g.q8.q, 1, M, N, g.q8.ldq, 32)) return cudaErrorInvalidValue;
    flags = STAGED;
  } else if (!((uintptr_t)g.out & 15) && g.ldo * es % 16 == 0 && make_map8(&mo, g.out, es, M, N, g.ldo, 32)) {
    flags = STAGED;
  }
  if (!Q8 && es == 2 && g.resid && !((uintptr_t)g.resid & 15) && g.ldr * es % 16 == 0 &&
      make_map8(&mr, g.resid, es, M, N, g.ldr, 32))
    flags |= RESID_TMA;
  const long long tiles = (long long)((M + 255) / 256) * ((N + 255) / 256);
  if (tiles > 0x7fffffff) return cudaErrorInvalidValue;
  const int pairs = sms / 2, grid = 2 * (int)(tiles < pairs ? tiles : pairs);
  const cudaError_t e = launch_pdl(k_gemm8_pair<T, Q8>, grid, P_THREADS, P_SMEM, s, ma, mw, mo, mr, M, N, K, flags, g);
  return e != cudaSuccess ? e : launched();
}

// The kernel and, for the split one, its rows of A to a tile and CTAs to a cluster: the
// least time of a model in us.  A tile's time is linear in its blocks of K, tiles run in
// waves over the SMs (two CTAs of the split kernel to an SM, each slower beside the
// other), and the cluster's meeting costs more the larger it is.  The constants are fitted
// to timings of all types and epilogues together, so the pairs' term is above their time
// with a plain bias (256 x 2048 x 8192: 33 us, 43 here).  At 130 other sizes (M 1 to 14566,
// N 48 to 12288, K 48 to 8192, all epilogues) the choice is 1.8% slower than the best one on
// average and more than 10% at eight, most of them with one to three blocks of K; 33% at
// worst (10585 x 69 x 317: 32 rows 12.8 us, pairs 9.7).  Either side of it, with a bias:
// 256 x 2048 x 8192 pairs 33 us, 64 rows and 4 CTAs 16.6; 512 x 2048 x 2048 pairs 12.8, 32
// rows 10.5; 1024 x 2048 x 2048 pairs 13.3, 64 rows 16.5.  (128 rows to a tile cost more in
// this model than 64 at any size: twice the room, shorter tiles; there is no such kernel.)
struct Plan {
  int bt, s;   // bt 0: CTA pairs
};
Plan plan8(int M, int N, int K, int sms) {
  const long long kb = (K + BK - 1) / BK, wt = (N + 127) / 128;
  const long long pt = (long long)((M + 255) / 256) * ((N + 255) / 256);
  Plan best = {0, 1};
  double least = (double)((pt + sms / 2 - 1) / (sms / 2)) * (0.549 * kb + 3.65) + 4.7;
  const int bts[3] = {16, 32, 64};
  const double one[3] = {0.321, 0.381, 0.365}, two[3] = {0.300, 0.467, 0.558}, fixed[3] = {1.73, 2.15, 5.57};
  const double meet[4] = {0, 0.27, 0.23, 0.44};
  for (int i = 0; i < 3; ++i) {
    if (i > 0 && bts[i - 1] >= M) break;
    const long long tiles = wt * ((M + bts[i] - 1) / bts[i]);
    for (int l = 0; l < 4 && (1 << l) <= kb; ++l) {
      const long long ctas = tiles << l, room = 2ll * sms;
      const bool shared = ctas > sms;
      const double t = (double)((ctas + room - 1) / room) * ((shared ? two : one)[i] * (double)((kb + (1 << l) - 1) >> l) + fixed[i]) +
                       2.0 + meet[l] + (shared ? 0.61 : 0.0) + 0.18 * std::min(1.0, (double)ctas / (double)room);
      if (t < least) {
        least = t;
        best = {bts[i], 1 << l};
      }
    }
  }
  return best;
}

template <class T, bool Q8>
cudaError_t gemm8_t(int M, int N, int K, const Gemm8Args& g, cudaStream_t s) {
  int sms = 0;
  const cudaError_t e = device_sms(&sms);
  if (e != cudaSuccess) return e;
  const Plan p = plan8(M, N, K, sms);
  switch (p.bt) {
    case 16: return launch_split<T, Q8, 16>(M, N, K, p.s, g, s);
    case 32: return launch_split<T, Q8, 32>(M, N, K, p.s, g, s);
    case 64: return launch_split<T, Q8, 64>(M, N, K, p.s, g, s);
    default: return launch_pair<T, Q8>(M, N, K, sms, g, s);
  }
}

}  // namespace

cudaError_t gemm8(DType dt, int M, int N, int K, const Gemm8Args& g, cudaStream_t s) {
  if (M <= 0) return cudaSuccess;
  if (!init_driver()) return cudaErrorNotSupported;
  if (dt == F32) return g.out ? gemm8_t<float, false>(M, N, K, g, s) : gemm8_t<float, true>(M, N, K, g, s);
  return g.out ? gemm8_t<bf16, false>(M, N, K, g, s) : gemm8_t<bf16, true>(M, N, K, g, s);
}

cudaError_t gemm8_watchdog_take(unsigned int* flags) {
  const unsigned int zero = 0;
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpyFromSymbol(flags, g_watchdog8, sizeof(*flags));
  if (e == cudaSuccess && *flags) e = cudaMemcpyToSymbol(g_watchdog8, &zero, sizeof(zero));
  return e;
}

cudaError_t gemm8_watchdog_probe(unsigned long long (&limit_ns)[2]) {
  k_gemm8_probe<<<1, 64>>>();
  cudaError_t e = launched();
  if (e == cudaSuccess) e = cudaMemcpyFromSymbol(limit_ns, g_probe_ns, sizeof(limit_ns));
  for (unsigned long long& t : limit_ns) t *= PROBE_PART;
  return e;
}

}  // namespace ff
