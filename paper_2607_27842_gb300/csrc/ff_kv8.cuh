// Declarations of the 8-bit key-value cache's operators and of the block norms, shared
// with their C entries, and how kernels address the cache (format: featfix_ops.h).
#pragma once

#include "featfix_ops.h"
#include "ff_common.cuh"
#include "ff_q8.cuh"

namespace ff {

typedef featfix_kv_cache KvCache;

constexpr int KV_DIM_MAX = 256;

struct KvRows {   // k and v in adjacent rows
  long long rows;
  const int* row_start;   // nullable: one row to a sequence
  void* k; long long ldk;
  void* v; long long ldv;
};
cudaError_t launch_kv_write(DType dt, const KvCache& c, const KvRows& r, cudaStream_t s);
cudaError_t launch_kv_read(DType dt, const KvCache& c, const KvRows& r, cudaStream_t s);

struct KvAttnArgs {
  const void* q; long long ldq;
  void* out; long long ldo;
  float* lse;   // nullable
  int q_heads;
  float scale;
  int window;   // 0: none
  void* ws;
};
// q_heads and heads come apart from the cache: the size is asked for before there is one
size_t kv_attention_workspace(int seqs, int q_heads, int heads, int dim, long long tokens);
cudaError_t launch_kv_attention(DType dt, const KvCache& c, const KvAttnArgs& a, cudaStream_t s);

constexpr int BLOCK_NORMS_COLS_MAX = 16384;   // what the registers of 256 threads hold
struct BlockNormsArgs {
  const void* y; long long ldy;
  const void* weight_after;                    // nullable
  const float* gate; long long gate_stride;    // nullable
  const void* x; long long ldx;                // nullable
  float resid_scale;
  void* sum; long long ldsum;                  // nullable
  const void* weight;                          // nullable
  const float* scale; long long scale_stride;  // nullable
  const float* shift; long long shift_stride;  // nullable
  int rpb;
  int norm_after, centered;
  float eps;
  void* out; long long ldo;                    // out and q8.q null: the sum alone
  Quant8Out q8;
};
cudaError_t launch_block_norms(DType dt, long long rows, int C, const BlockNormsArgs& a, cudaStream_t s);

// Division of numbers below 2^31 by one that the host knows: a product's upper half.
struct Div {
  unsigned m, s;
  void by(unsigned d) {
    for (s = 0; (1ull << s) < d; ++s) {}
    m = (unsigned)(((1ull << 32) * ((1ull << s) - d)) / d + 1);
  }
  __device__ __forceinline__ int of(unsigned n) const { return (int)((__umulhi(m, n) + n) >> s); }
};

// Tokens of a sequence, by its place in lens: what the table can hold at most.
__device__ __forceinline__ int kv_len(const KvCache& c, int len) {
  const long long most = (long long)c.table_pages * c.page_size;
  return (int)max(0ll, min((long long)len, most));
}

// What a scale stands for: infinities and negative numbers are NaN (featfix_ops.h).
__device__ __forceinline__ float kv_scale(float s) {
  return s >= 0.f && s < __int_as_float(0x7f800000) ? s : __int_as_float(0x7fffffff);
}

}  // namespace ff
