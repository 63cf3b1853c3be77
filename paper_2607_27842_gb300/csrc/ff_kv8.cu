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
// First rows and lengths of the sequences, by a block in shared memory where there are not too many: one
// wait for memory instead of one for every halving of the search and one for the length (8000 rows of 19
// sequences 8.4 -> 6 us).
constexpr int SEQS_HELD = 512;
struct Sequences {
  int start[SEQS_HELD + 1], len[SEQS_HELD];
};
__device__ __forceinline__ bool hold(const KvCache& c, const int* row_start, Sequences& q) {
  if (!row_start || c.seqs > SEQS_HELD) return false;
  for (int i = threadIdx.x; i <= c.seqs; i += blockDim.x) {
    q.start[i] = row_start[i];
    if (i < c.seqs) q.len[i] = kv_len(c, i);
  }
  __syncthreads();
  return true;
}
__device__ __forceinline__ Place place_of(const KvCache& c, const int* row_start, const Sequences* held, long long row,
                                          const Div& page_size) {
  int b = (int)row, back = 1;   // rows from this one to the sequence's last
  if (row_start) {
    const int* start = held ? held->start : row_start;
    // the last sequence that starts at or before the row (empty ones end where they start)
    int lo = 0, hi = c.seqs;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (start[mid] <= row) lo = mid + 1;
      else hi = mid;
    }
    b = lo - 1;
    const int end = b < 0 ? 0 : start[b + 1];
    if (row >= end) return {-1, 0, true};
    back = end - (int)row;
  }
  const int t = (held ? held->len[b] : kv_len(c, b)) - back;
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

// L lanes to a head of a row, sixteen columns to a lane, U such heads to a lane, all loads of which are
// under way before the first is used.  Bound by instruction issue before it was by memory: hence sixteen
// columns (eight: 14566 x 16 heads of 128 in bf16 49 us, half of its instructions addresses and the
// maximum's exchange) and 32-bit strides.
template <class T, bool VEC, int L, int U>
__global__ void __launch_bounds__(256) k_kv_write(const __grid_constant__ KvCache c, const __grid_constant__ KvRows r,
                                                  const Div heads, const Div page_size) {
  constexpr int G = 256 / L;
  __shared__ Sequences sequences;
  const int lane = threadIdx.x % L, col = 16 * lane, n = min(2, max(0, c.head_dim - col) / 8);   // eights of this lane
  pdl_trigger();
  pdl_wait();
  Eight<T, VEC> x[U][2][2];
  int head[U];
  long long row[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long item = ((long long)blockIdx.x * U + u) * G + threadIdx.x / L;
    row[u] = item >> 31 ? item / c.heads : heads.of((unsigned)item);
    head[u] = (int)(item - row[u] * c.heads);
    const int at = head[u] * c.head_dim + col;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x[u][0][i].zero();
      x[u][1][i].zero();
      if (row[u] < r.rows && i < n) {
        x[u][0][i].load(reinterpret_cast<const T*>(r.k) + row[u] * r.ldk + at + 8 * i);
        x[u][1][i].load(reinterpret_cast<const T*>(r.v) + row[u] * r.ldv + at + 8 * i);
      }
    }
  }
  const Sequences* held = hold(c, r.row_start, sequences) ? &sequences : nullptr;
  Place p[U];
#pragma unroll
  for (int u = 0; u < U; ++u) p[u] = row[u] < r.rows ? place_of(c, r.row_start, held, row[u], page_size) : Place{-1, 0, true};
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      float v[16];
      x[u][kv][0].get(v);
      x[u][kv][1].get(v + 8);
      float m = amax16<T, VEC>(x[u][kv], v);
#pragma unroll
      for (int o = L / 2; o; o >>= 1) m = max_abs(m, __shfl_xor_sync(0xffffffffu, m, o));
      if (p[u].page < 0 || n == 0) continue;
      const float s = q8_scale(__float_as_uint(m)), inv = q8_inv(s);
      uint8_t* q = reinterpret_cast<uint8_t*>(kv ? c.v : c.k) + place_at(kv ? c.v_stride : c.k_stride, p[u], head[u]) + col;
      const f32x2 i2 = f2u(inv, inv);
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x2 a = fmul2(f2u(v[4 * i], v[4 * i + 1]), i2), b = fmul2(f2u(v[4 * i + 2], v[4 * i + 3]), i2);
        w[i] = to_e4m3x4(lo_f(a), hi_f(a), lo_f(b), hi_f(b));
      }
      if (n == 2) *reinterpret_cast<uint4*>(q) = make_uint4(w[0], w[1], w[2], w[3]);
      else *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
      if (lane == 0) (kv ? c.v_scale : c.k_scale)[place_at(kv ? c.v_scale_stride : c.k_scale_stride, p[u], head[u])] = s;
    }
}

// four e4m3 bytes as floats
__device__ __forceinline__ void from_e4m3x4(uint32_t u, float* v) {
  const __half2_raw a = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(u & 0xffff), __NV_E4M3);
  const __half2_raw b = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(u >> 16), __NV_E4M3);
  const float2 x = __half22float2(a), y = __half22float2(b);
  v[0] = x.x, v[1] = x.y, v[2] = y.x, v[3] = y.y;
}

// L threads to a head of a row, as many columns to each as 16 bytes of the result hold (so that
// adjacent lanes write adjacent vectors), U such heads to a thread, all loads under way before the
// first is used.  Bound by memory.
template <class T, bool VEC, int L, int U>
__global__ void __launch_bounds__(256) k_kv_read(const __grid_constant__ KvCache c, const __grid_constant__ KvRows r,
                                                 const Div heads, const Div page_size) {
  constexpr int G = 256 / L;
  constexpr int E = VecN<T>::n;
  const int lane = threadIdx.x % L, col = E * lane;
  __shared__ Sequences sequences;
  pdl_trigger();
  pdl_wait();
  const Sequences* held = hold(c, r.row_start, sequences) ? &sequences : nullptr;
  if (col >= c.head_dim) return;
  Place p[U];
  int head[U];
  long long row[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long item = ((long long)blockIdx.x * U + u) * G + threadIdx.x / L;
    row[u] = item >> 31 ? item / c.heads : heads.of((unsigned)item);
    head[u] = (int)(item - row[u] * c.heads);
    p[u] = row[u] < r.rows ? place_of(c, r.row_start, held, row[u], page_size) : Place{-1, 0, true};
  }
  uint32_t q[U][2][E / 4];
  float s[U][2];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
#pragma unroll
      for (int i = 0; i < E / 4; ++i) q[u][kv][i] = 0;
      s[u][kv] = 0.f;
      if (p[u].page < 0) continue;
      const uint8_t* at = reinterpret_cast<const uint8_t*>(kv ? c.v : c.k) + place_at(kv ? c.v_stride : c.k_stride, p[u], head[u]) + col;
      if constexpr (E == 8) {
        const uint2 v = *reinterpret_cast<const uint2*>(at);
        q[u][kv][0] = v.x, q[u][kv][E / 4 - 1] = v.y;
      } else {
        q[u][kv][0] = *reinterpret_cast<const uint32_t*>(at);
      }
      s[u][kv] = (kv ? c.v_scale : c.k_scale)[place_at(kv ? c.v_scale_stride : c.k_scale_stride, p[u], head[u])];
    }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (p[u].of_none) continue;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      float x[E];
#pragma unroll
      for (int i = 0; i < E / 4; ++i) from_e4m3x4(q[u][kv][i], x + 4 * i);
      const float f = kv_scale(s[u][kv]);
#pragma unroll
      for (int i = 0; i < E; ++i) x[i] *= f;
      store_vec<T, VEC>(reinterpret_cast<T*>(kv ? r.v : r.k) + row[u] * (kv ? r.ldv : r.ldk) + (long long)head[u] * c.head_dim + col, x);
    }
  }
}

template <class T, bool VEC, bool WRITE, int L, int U> cudaError_t kv_rows_u(const KvCache& c, const KvRows& r, cudaStream_t s) {
  const long long per = 256 / L * U, grid = (r.rows * c.heads + per - 1) / per;
  if (grid > 0x7fffffff) return cudaErrorInvalidValue;
  Div heads, page_size;
  heads.by(c.heads);
  page_size.by(c.page_size);
  const cudaError_t e = WRITE ? launch_pdl(k_kv_write<T, VEC, L, U>, (unsigned)grid, 256, 0, s, c, r, heads, page_size)
                              : launch_pdl(k_kv_read<T, VEC, L, U>, (unsigned)grid, 256, 0, s, c, r, heads, page_size);
  return e != cudaSuccess ? e : launched();
}
template <class T, bool VEC, bool WRITE, int L> cudaError_t kv_rows_l(const KvCache& c, const KvRows& r, cudaStream_t s) {
  // several heads to a lane where two blocks of them for every SM remain
  // (read 14566 x 16 heads of 128 in bf16: 32.2 us with two, 33.6 with four, 44.8 with eight)
  constexpr int U = WRITE && sizeof(T) == 4 ? 1 : 2;
  if (U > 1 && r.rows * c.heads >= 152ll * 2 * U * (256 / L)) return kv_rows_u<T, VEC, WRITE, L, U>(c, r, s);
  return kv_rows_u<T, VEC, WRITE, L, 1>(c, r, s);
}
template <class T, bool VEC, bool WRITE> cudaError_t kv_rows_v(const KvCache& c, const KvRows& r, cudaStream_t s) {
  constexpr int L = WRITE ? 4 : 64 / VecN<T>::n;   // threads to 64 columns
  return c.head_dim <= 64 ? kv_rows_l<T, VEC, WRITE, L>(c, r, s)
         : c.head_dim <= 128 ? kv_rows_l<T, VEC, WRITE, 2 * L>(c, r, s) : kv_rows_l<T, VEC, WRITE, 4 * L>(c, r, s);
}
template <class T, bool WRITE> cudaError_t kv_rows(const KvCache& c, const KvRows& r, cudaStream_t s) {
  const auto al = [](const void* p, long long ld) { return !((uintptr_t)p & 15) && ld % (16 / (int)sizeof(T)) == 0; };
  return al(r.k, r.ldk) && al(r.v, r.ldv) ? kv_rows_v<T, true, WRITE>(c, r, s) : kv_rows_v<T, false, WRITE>(c, r, s);
}

}  // namespace

cudaError_t launch_kv_write(DType dt, const KvCache& c, const KvRows& r, cudaStream_t s) {
  return dt == F32 ? kv_rows<float, true>(c, r, s) : kv_rows<bf16, true>(c, r, s);
}
cudaError_t launch_kv_read(DType dt, const KvCache& c, const KvRows& r, cudaStream_t s) {
  return dt == F32 ? kv_rows<float, false>(c, r, s) : kv_rows<bf16, false>(c, r, s);
}

}  // namespace ff
