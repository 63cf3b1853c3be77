// Key-value cache in 8 bits: new tokens into their pages, and tokens back out of them
// (format and formulas: featfix_ops.h).  Both are bound by memory: every element is read
// once into registers and written once.
#include "ff_kv8.cuh"

#include <algorithm>

namespace ff {

namespace {

// Eight elements of a head, the share of one lane: in 16-byte vectors, or one by one
// where rows start off them.
template <class T, bool VEC> __device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  if constexpr (!VEC) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f(p[i]);
  } else if constexpr (sizeof(T) == 2) {
    ld16(p, v);
  } else {
    float a[4], b[4];
    ld16(p, a);
    ld16(p + 4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[i + 4] = b[i];
  }
}
template <class T, bool VEC> __device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  if constexpr (!VEC) {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = from_f<T>(v[i]);
  } else if constexpr (sizeof(T) == 2) {
    st16(p, v);
  } else {
    const float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
    st16(p, a);
    st16(p + 4, b);
  }
}

// Sequence and token of a row of the call; false where the row has none.
struct Token {
  int b, t;
};
__device__ __forceinline__ bool token_of(const KvCache& c, const int* row_start, long long row, Token* o) {
  if (!row_start) {
    *o = {(int)row, kv_len(c, (int)row) - 1};
    return true;
  }
  // the last sequence that starts at or before the row (empty ones end where they start)
  int lo = 0, hi = c.seqs;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (row_start[mid] <= row) lo = mid + 1;
    else hi = mid;
  }
  const int b = lo - 1;
  if (b < 0) return false;
  const int end = row_start[b + 1];
  if (row >= end) return false;
  *o = {b, (int)(kv_len(c, b) - (end - row))};
  return true;
}

// L lanes to a head of one row.
template <class T, bool VEC, int L>
__global__ void __launch_bounds__(256) k_kv_write(const __grid_constant__ KvCache c, const __grid_constant__ KvRows r) {
  const int lane = threadIdx.x % L, col = 8 * lane;
  const long long item = (long long)blockIdx.x * (256 / L) + threadIdx.x / L;
  const long long row = item / c.heads;
  const int head = (int)(item - row * c.heads);
  pdl_trigger();
  pdl_wait();
  Token tk;
  int page = -1;
  if (row < r.rows && token_of(c, r.row_start, row, &tk) && tk.t >= 0) page = kv_page(c, tk.b, tk.t);
  const int slot = page < 0 ? 0 : tk.t % c.page_size;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (page >= 0 && col < c.head_dim)
      load8<T, VEC>(reinterpret_cast<const T*>(kv ? r.v : r.k) + row * (kv ? r.ldv : r.ldk) + (long long)head * c.head_dim + col, x);
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max_abs(m, x[i]);
#pragma unroll
    for (int o = L / 2; o; o >>= 1) m = max_abs(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (page < 0 || col >= c.head_dim) continue;
    const float s = q8_scale(__float_as_uint(m)), inv = q8_inv(s);
    const long long* st = kv ? c.v_stride : c.k_stride;
    uint8_t* q = reinterpret_cast<uint8_t*>(kv ? c.v : c.k) + page * st[0] + slot * st[1] + head * st[2] + col;
    *reinterpret_cast<uint2*>(q) = make_uint2(to_e4m3x4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv),
                                              to_e4m3x4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv));
    const long long* ss = kv ? c.v_scale_stride : c.k_scale_stride;
    if (lane == 0) (kv ? c.v_scale : c.k_scale)[page * ss[0] + slot * ss[1] + head * ss[2]] = s;
  }
}

// four e4m3 bytes as floats
__device__ __forceinline__ void from_e4m3x4(uint32_t u, float* v) {
  const __half2_raw a = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(u & 0xffff), __NV_E4M3);
  const __half2_raw b = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(u >> 16), __NV_E4M3);
  const float2 x = __half22float2(a), y = __half22float2(b);
  v[0] = x.x, v[1] = x.y, v[2] = y.x, v[3] = y.y;
}

template <class T, bool VEC, int L>
__global__ void __launch_bounds__(256) k_kv_read(const __grid_constant__ KvCache c, const __grid_constant__ KvRows r) {
  const int lane = threadIdx.x % L, col = 8 * lane;
  const long long item = (long long)blockIdx.x * (256 / L) + threadIdx.x / L;
  const long long row = item / c.heads;
  const int head = (int)(item - row * c.heads);
  pdl_trigger();
  pdl_wait();
  Token tk;
  if (row >= r.rows || col >= c.head_dim || !token_of(c, r.row_start, row, &tk)) return;
  const int page = tk.t < 0 ? -1 : kv_page(c, tk.b, tk.t);
  const int slot = page < 0 ? 0 : tk.t % c.page_size;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (page >= 0) {
      const long long* st = kv ? c.v_stride : c.k_stride;
      const uint8_t* q = reinterpret_cast<const uint8_t*>(kv ? c.v : c.k) + page * st[0] + slot * st[1] + head * st[2] + col;
      const long long* ss = kv ? c.v_scale_stride : c.k_scale_stride;
      const float s = kv_scale((kv ? c.v_scale : c.k_scale)[page * ss[0] + slot * ss[1] + head * ss[2]]);
      const uint2 u = *reinterpret_cast<const uint2*>(q);
      from_e4m3x4(u.x, x);
      from_e4m3x4(u.y, x + 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= s;
    }
    store8<T, VEC>(reinterpret_cast<T*>(kv ? r.v : r.k) + row * (kv ? r.ldv : r.ldk) + (long long)head * c.head_dim + col, x);
  }
}

template <class T, bool VEC, bool WRITE, int L> cudaError_t kv_rows_l(const KvCache& c, const KvRows& r, cudaStream_t s) {
  const long long grid = (r.rows * c.heads + 256 / L - 1) / (256 / L);
  if (grid > 0x7fffffff) return cudaErrorInvalidValue;
  const cudaError_t e = WRITE ? launch_pdl(k_kv_write<T, VEC, L>, (unsigned)grid, 256, 0, s, c, r)
                              : launch_pdl(k_kv_read<T, VEC, L>, (unsigned)grid, 256, 0, s, c, r);
  return e != cudaSuccess ? e : launched();
}
template <class T, bool VEC, bool WRITE> cudaError_t kv_rows_v(const KvCache& c, const KvRows& r, cudaStream_t s) {
  return c.head_dim <= 64 ? kv_rows_l<T, VEC, WRITE, 8>(c, r, s)
         : c.head_dim <= 128 ? kv_rows_l<T, VEC, WRITE, 16>(c, r, s) : kv_rows_l<T, VEC, WRITE, 32>(c, r, s);
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
