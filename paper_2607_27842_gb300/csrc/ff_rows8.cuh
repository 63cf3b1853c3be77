// How the row kernels of the 8-bit layers go over a row: warps have adjacent 128-column blocks
// of it, a lane four columns of each.
#pragma once

#include "ff_q8.cuh"

namespace ff {

// Four elements of a lane's share of a 128-column block, as two fp32 pairs: adjacent
// columns 4 lane .. in one vector where rows allow it, columns lane, lane + 32, ..
// otherwise.  Pointers are to the lane's first column (at()), n the columns from
// there to the row's end.
template <class T, bool VEC> struct Four;
template <bool VEC> __device__ __forceinline__ int at(int lane) { return VEC ? 4 * lane : lane; }
template <> struct Four<float, true> {
  ulonglong2 r;
  __device__ __forceinline__ void load(const float* p, int) { r = *reinterpret_cast<const ulonglong2*>(p); }
  __device__ __forceinline__ void get(f32x2 (&v)[2]) const { v[0] = r.x; v[1] = r.y; }
  static __device__ __forceinline__ void store(float* p, int, const f32x2 (&v)[2]) {
    *reinterpret_cast<ulonglong2*>(p) = make_ulonglong2(v[0], v[1]);
  }
};
template <> struct Four<bf16, true> {
  uint2 r;
  __device__ __forceinline__ void load(const bf16* p, int) { r = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void get(f32x2 (&v)[2]) const { v[0] = bf2u(r.x); v[1] = bf2u(r.y); }
  static __device__ __forceinline__ void store(bf16* p, int, const f32x2 (&v)[2]) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(lo_f(v[0]), hi_f(v[0])), b = __floats2bfloat162_rn(lo_f(v[1]), hi_f(v[1]));
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
  }
};
template <class T> struct Four<T, false> {
  T r[4];
  __device__ __forceinline__ void load(const T* p, int n) {
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = 32 * k < n ? p[32 * k] : from_f<T>(0.f);
  }
  __device__ __forceinline__ void get(f32x2 (&v)[2]) const {
    v[0] = f2u(to_f(r[0]), to_f(r[1]));
    v[1] = f2u(to_f(r[2]), to_f(r[3]));
  }
  static __device__ __forceinline__ void store(T* p, int n, const f32x2 (&v)[2]) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (32 * k < n) p[32 * k] = from_f<T>(k & 1 ? hi_f(v[k / 2]) : lo_f(v[k / 2]));
  }
};
// the four as e4m3
template <bool VEC>
__device__ __forceinline__ void store8(uint8_t* p, int n, const f32x2 (&v)[2], float inv) {
  const f32x2 i2 = f2u(inv, inv), a = fmul2(v[0], i2), b = fmul2(v[1], i2);
  const uint32_t c = to_e4m3x4(lo_f(a), hi_f(a), lo_f(b), hi_f(b));
  if (VEC) {
    *reinterpret_cast<uint32_t*>(p) = c;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (32 * k < n) p[32 * k] = (uint8_t)(c >> (8 * k));
  }
}
__device__ __forceinline__ float amax4(const f32x2 (&v)[2]) {
  return max_abs(max_abs(lo_f(v[0]), hi_f(v[0])), max_abs(lo_f(v[1]), hi_f(v[1])));
}

// Whether a row pointer and stride keep vectors of four elements aligned.
template <class T> inline bool al4(const void* p, long long ld) {
  return !((uintptr_t)p & (4 * sizeof(T) - 1)) && ld % 4 == 0;
}

}  // namespace ff
