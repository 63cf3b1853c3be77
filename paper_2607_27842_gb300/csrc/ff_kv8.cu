// Key-value cache in 8 bits: new tokens into their pages, and tokens back out of them
// (format and formulas: featfix_ops.h).  Both are bound by memory: every element is read
// once into registers and written once.
#include "ff_kv8.cuh"

#include <algorithm>

namespace ff {

namespace {

// Eight elements of a head, the share of one lane: in 16-byte vectors, or one by one
// where rows start off them.  As they are in memory, so that loads wait for nothing.
template <class T, bool VEC> struct Eight {
  T r[8];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = p[i];
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = from_f<T>(0.f);
  }
  __device__ __forceinline__ void get(float* v) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f(r[i]);
  }
};
template <class T> struct Eight<T, true> {
  uint4 r[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r[i] = make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void get(float* v) const {
    if constexpr (sizeof(T) == 2) {
      float u[8];
      unpack16(r[0], u);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = u[i];
    } else {
      const uint32_t w[8] = {r[0].x, r[0].y, r[0].z, r[0].w, r[1].x, r[1].y, r[1].z, r[1].w};
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
    }
  }
};
// As many elements as 16 bytes hold, in a vector or one by one.
template <class T, bool VEC> __device__ __forceinline__ void store_vec(T* p, const float (&v)[VecN<T>::n]) {
  if constexpr (VEC) {
    st16(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < VecN<T>::n; ++i) p[i] = from_f<T>(v[i]);
  }
}

// Where a row's token lies: page (-1: nowhere) and slot; of_none: the row is of no sequence.
struct Place {
  int page, slot;
  bool of_none;
};
// (by a whole warp)
__device__ __forceinline__ Place place_of(const KvCache& c, const int* row_start, long long row, const Div& page_size) {
  int b = (int)row, back = 1;   // rows from this one to the sequence's last
  if (row_start) {
    // the last sequence that starts at or before the row (empty ones end where they start), by 32 starts at
    // a time: one wait for memory up to 31 sequences, two up to 1023
    const int lane = threadIdx.x & 31;
    int lo = 0, n = c.seqs + 1;
    while (n > 1) {
      const int step = (n + 31) / 32, at = lane * step;
      const int k = __popc(__ballot_sync(0xffffffffu, at < n && row_start[lo + min(at, n - 1)] <= row));
      if (k == 0) return {-1, 0, true};
      lo += (k - 1) * step;
      n = min(step, n - (k - 1) * step);
    }
    if (lo == c.seqs) return {-1, 0, true};
    b = lo;
    back = row_start[b + 1] - (int)row;
    if (back <= 0) return {-1, 0, true};   // (starts that do not rise)
  }
  const int t = kv_len(c, c.lens[b]) - back;
  if (t < 0) return {-1, 0, false};
  const int n = page_size.of((unsigned)t), page = c.table[b * c.ld_table + n];
  return {(unsigned)page < (unsigned)c.pages ? page : -1, t - n * c.page_size, false};
}

// Where a place starts (strides are below 2^32: products of 32 bits).
__device__ __forceinline__ unsigned long long place_at(const long long (&st)[3], const Place& p, int head) {
  return (unsigned long long)(unsigned)p.page * (unsigned)st[0] + (unsigned long long)(unsigned)p.slot * (unsigned)st[1] +
         (unsigned long long)(unsigned)head * (unsigned)st[2];
}

// Largest magnitude of a lane's sixteen elements: bf16 in pairs, as they are in memory.
template <class T, bool VEC> __device__ __forceinline__ float amax16(const Eight<T, VEC> (&e)[2], const float (&v)[16]) {
  if constexpr (VEC && sizeof(T) == 2) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t w[4] = {e[i].r[0].x, e[i].r[0].y, e[i].r[0].z, e[i].r[0].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) asm("max.NaN.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(w[k]));
    }
    return max_abs(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  } else {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max_abs(m, v[i]);
    return m;
  }
}

// A warp to a row, or to an equal part of its heads: a row's place is looked up once, while its first
// columns are under way.  L lanes to a head, sixteen columns to a lane.  Bound by instruction issue
// before it was by memory: hence sixteen columns (eight, and a look-up for every head: 14566 x 16 heads of
// 128 in bf16 46 us) and 32-bit strides.  Now 30.6 us, 5.9 TB/s, and 45.7 from fp32, 6.6 TB/s; one token of 4
// heads 1.9 us in a graph.
template <class T, bool VEC, int L>
__global__ void __launch_bounds__(256) k_kv_write(const __grid_constant__ KvCache c, const __grid_constant__ KvRows r,
                                                  const Div parts_by, int parts, int per, const Div page_size) {
  const int lane = threadIdx.x & 31, col = 16 * (lane % L), n = min(2, max(0, c.head_dim - col) / 8);   // eights of this lane
  const long long warp = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const long long row = warp >> 31 ? warp / parts : parts_by.of((unsigned)warp);
  const int first = (int)(warp - row * parts) * per, end = min(c.heads, first + per);
  pdl_trigger();
  pdl_wait();
  if (row >= r.rows) return;
  const T* from[2] = {reinterpret_cast<const T*>(r.k) + row * r.ldk + col, reinterpret_cast<const T*>(r.v) + row * r.ldv + col};
  Place p = {-1, 0, true};
  for (int h0 = first; h0 < end; h0 += 32 / L) {
    const int head = h0 + lane / L;
    const bool in = head < end && n > 0;
    Eight<T, VEC> x[2][2];
#pragma unroll
    for (int kv = 0; kv < 2; ++kv)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x[kv][i].zero();
        if (in && i < n) x[kv][i].load(from[kv] + head * c.head_dim + 8 * i);
      }
    if (h0 == first) {
      p = place_of(c, r.row_start, row, page_size);
      // (one place for all lanes, unless lengths or table change meanwhile: then too the warp goes on together)
      if (!__any_sync(0xffffffffu, p.page >= 0)) return;
    }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      float v[16];
      x[kv][0].get(v);
      x[kv][1].get(v + 8);
      float m = amax16<T, VEC>(x[kv], v);
#pragma unroll
      for (int o = L / 2; o; o >>= 1) m = max_abs(m, __shfl_xor_sync(0xffffffffu, m, o));
      if (!in || p.page < 0) continue;
      const float s = q8_scale(__float_as_uint(m)), inv = q8_inv(s);
      uint8_t* q = reinterpret_cast<uint8_t*>(kv ? c.v : c.k) + place_at(kv ? c.v_stride : c.k_stride, p, head) + col;
      const f32x2 i2 = f2u(inv, inv);
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x2 a = fmul2(f2u(v[4 * i], v[4 * i + 1]), i2), b = fmul2(f2u(v[4 * i + 2], v[4 * i + 3]), i2);
        w[i] = to_e4m3x4(lo_f(a), hi_f(a), lo_f(b), hi_f(b));
      }
      if (n == 2) *reinterpret_cast<uint4*>(q) = make_uint4(w[0], w[1], w[2], w[3]);
      else *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
      if (col == 0) (kv ? c.v_scale : c.k_scale)[place_at(kv ? c.v_scale_stride : c.k_scale_stride, p, head)] = s;
    }
  }
}

// four e4m3 bytes as floats
__device__ __forceinline__ void from_e4m3x4(uint32_t u, float* v) {
  const __half2_raw a = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(u & 0xffff), __NV_E4M3);
  const __half2_raw b = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(u >> 16), __NV_E4M3);
  const float2 x = __half22float2(a), y = __half22float2(b);
  v[0] = x.x, v[1] = x.y, v[2] = y.x, v[3] = y.y;
}

// A warp to a row, or to an equal part of its vectors (as many columns as 16 bytes of the result hold, so
// that adjacent lanes write adjacent vectors): a row's place is looked up once.  U vectors of k and of v
// are under way at a time.  Bound by memory: 14566 x 16 heads of 128 30.0 us in bf16, 6.0 TB/s, 49.9 in fp32.
template <class T, bool VEC, int U>
__global__ void __launch_bounds__(256) k_kv_read(const __grid_constant__ KvCache c, const __grid_constant__ KvRows r,
                                                 const Div parts_by, int parts, int per, const Div dim_by, const Div page_size) {
  constexpr int E = VecN<T>::n;
  const int lane = threadIdx.x & 31;
  const long long warp = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const long long row = warp >> 31 ? warp / parts : parts_by.of((unsigned)warp);
  const int first = (int)(warp - row * parts) * per + lane, all = c.heads * (c.head_dim / E), end = min(all, first - lane + per);
  pdl_trigger();
  pdl_wait();
  if (row >= r.rows) return;
  const Place p = place_of(c, r.row_start, row, page_size);
  if (p.of_none) return;
  const uint8_t* from[2] = {reinterpret_cast<const uint8_t*>(c.k) + place_at(c.k_stride, p, 0),
                            reinterpret_cast<const uint8_t*>(c.v) + place_at(c.v_stride, p, 0)};
  const float* scale[2] = {c.k_scale + place_at(c.k_scale_stride, p, 0), c.v_scale + place_at(c.v_scale_stride, p, 0)};
  const unsigned step[2] = {(unsigned)c.k_stride[2], (unsigned)c.v_stride[2]};
  const unsigned scale_step[2] = {(unsigned)c.k_scale_stride[2], (unsigned)c.v_scale_stride[2]};
  T* to[2] = {reinterpret_cast<T*>(r.k) + row * r.ldk, reinterpret_cast<T*>(r.v) + row * r.ldv};
  for (int i = first; i < end; i += 32 * U) {
    uint32_t q[U][2][E / 4];
    float s[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = (i + 32 * u) * E, head = dim_by.of((unsigned)at), col = at - head * c.head_dim;
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        s[u][kv] = 0.f;
#pragma unroll
        for (int k = 0; k < E / 4; ++k) q[u][kv][k] = 0;
        if (p.page < 0 || i + 32 * u >= end) continue;
        const uint8_t* b = from[kv] + (unsigned long long)(unsigned)head * step[kv] + col;
        if constexpr (E == 8) {
          const uint2 v = *reinterpret_cast<const uint2*>(b);
          q[u][kv][0] = v.x, q[u][kv][E / 4 - 1] = v.y;
        } else {
          q[u][kv][0] = *reinterpret_cast<const uint32_t*>(b);
        }
        s[u][kv] = scale[kv][(unsigned long long)(unsigned)head * scale_step[kv]];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + 32 * u >= end) break;
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        float x[E];
#pragma unroll
        for (int k = 0; k < E / 4; ++k) from_e4m3x4(q[u][kv][k], x + 4 * k);
        const float f = kv_scale(s[u][kv]);
#pragma unroll
        for (int k = 0; k < E; ++k) x[k] *= f;
        store_vec<T, VEC>(to[kv] + (i + 32 * u) * E, x);
      }
    }
  }
}

// Steps of a row's loop that go to a warp: as many as leave WARPS_HELD warps to an SM.
constexpr int WARPS_HELD = 128;   // (14566 x 16 heads of 128 in bf16, read: 31.9 us with 64, 29.9 with 128, 30.6 with 256)
long long steps_to_warp(long long rows, long long steps) {
  return std::max(1ll, std::min(steps, rows * steps / (152ll * WARPS_HELD)));
}
template <class T, bool VEC, int L> cudaError_t kv_write_l(const KvCache& c, const KvRows& r, cudaStream_t s) {
  const long long steps = (c.heads + 32 / L - 1) / (32 / L), n = steps_to_warp(r.rows, steps), parts = (steps + n - 1) / n;
  const long long grid = (r.rows * parts + 7) / 8;
  if (grid > 0x7fffffff) return cudaErrorInvalidValue;
  Div parts_by, page_size;
  parts_by.by((unsigned)parts);
  page_size.by(c.page_size);
  const cudaError_t e = launch_pdl(k_kv_write<T, VEC, L>, (unsigned)grid, 256, 0, s, c, r, parts_by, (int)parts, (int)(32 / L * n), page_size);
  return e != cudaSuccess ? e : launched();
}
template <class T, bool VEC> cudaError_t kv_write(const KvCache& c, const KvRows& r, cudaStream_t s) {
  return c.head_dim <= 64 ? kv_write_l<T, VEC, 4>(c, r, s)
         : c.head_dim <= 128 ? kv_write_l<T, VEC, 8>(c, r, s) : kv_write_l<T, VEC, 16>(c, r, s);
}
template <class T, bool VEC> cudaError_t kv_read(const KvCache& c, const KvRows& r, cudaStream_t s) {
  constexpr int U = 2;
  const long long all = (long long)c.heads * (c.head_dim / VecN<T>::n), steps = (all + 32 * U - 1) / (32 * U);
  const long long n = steps_to_warp(r.rows, steps), parts = (steps + n - 1) / n;
  const long long grid = (r.rows * parts + 7) / 8;
  if (grid > 0x7fffffff) return cudaErrorInvalidValue;
  Div parts_by, dim_by, page_size;
  parts_by.by((unsigned)parts);
  dim_by.by(c.head_dim);
  page_size.by(c.page_size);
  const cudaError_t e = launch_pdl(k_kv_read<T, VEC, U>, (unsigned)grid, 256, 0, s, c, r, parts_by, (int)parts, (int)(32 * U * n), dim_by, page_size);
  return e != cudaSuccess ? e : launched();
}
template <class T, bool WRITE> cudaError_t kv_rows(const KvCache& c, const KvRows& r, cudaStream_t s) {
  const auto al = [](const void* p, long long ld) { return !((uintptr_t)p & 15) && ld % (16 / (int)sizeof(T)) == 0; };
  const bool vec = al(r.k, r.ldk) && al(r.v, r.ldv);
  if constexpr (WRITE) return vec ? kv_write<T, true>(c, r, s) : kv_write<T, false>(c, r, s);
  else return vec ? kv_read<T, true>(c, r, s) : kv_read<T, false>(c, r, s);
}

}  // namespace

cudaError_t launch_kv_write(DType dt, const KvCache& c, const KvRows& r, cudaStream_t s) {
  return dt == F32 ? kv_rows<float, true>(c, r, s) : kv_rows<bf16, true>(c, r, s);
}
cudaError_t launch_kv_read(DType dt, const KvCache& c, const KvRows& r, cudaStream_t s) {
  return dt == F32 ? kv_rows<float, false>(c, r, s) : kv_rows<bf16, false>(c, r, s);
}

}  // namespace ff
