// C ABI of include/featfix_ops.h: the hot-path kernels on caller buffers.
#include "featfix_ops.h"
#include "ff_common.cuh"
#include "ff_kv8.cuh"
#include "ff_q8.cuh"

#include <math.h>

#include <initializer_list>

using namespace ff;

namespace {

bool dt_ok(int dt) { return dt == FEATFIX_DTYPE_F32 || dt == FEATFIX_DTYPE_BF16; }
bool al16(const void* p) { return ((uintptr_t)p & 15) == 0; }
// largest dimension of the 8-bit layers: rounding up to a tile stays an int
constexpr long long DIM_MAX = 0x7fffff00;
// every given pointer on its element's boundary
bool el_al(int dt, std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if ((uintptr_t)p & (dt == FEATFIX_DTYPE_F32 ? 3 : 1)) return false;
  return true;
}
// an 8-bit tensor of `width` columns with at least `scales` scales to a row of them
bool q8_ok(const Quant8Out& t, long long width, long long scales) {
  return t.q && t.scale && al16(t.q) && t.ldq >= width && t.ldq % 16 == 0 && !((uintptr_t)t.scale & 3) &&
         t.lds >= scales;
}
featfix_status st(cudaError_t e) {
  if (e == cudaSuccess) return FEATFIX_OK;
  if (e == cudaErrorInvalidValue) return FEATFIX_ERR_INVALID_ARG;
  if (e == cudaErrorNotSupported) return FEATFIX_ERR_UNSUPPORTED;
  return FEATFIX_ERR_CUDA;
}

constexpr int PAGE_MAX = 1 << 24;
// Places at least `width` (in units of `unit`) apart along each dimension that has more than one.
bool strides_ok(const featfix_kv_cache& c, const long long (&st)[3], long long width, int unit) {
  const int n[3] = {c.pages, c.page_size, c.heads};
  for (int i = 0; i < 3; ++i)
    if (n[i] > 1 && (st[i] < width || st[i] % unit || st[i] > 0xffffffffll)) return false;
  return true;
}
bool cache_ok(const featfix_kv_cache* c) {
  if (!c || c->pages <= 0 || c->page_size <= 0 || c->page_size > PAGE_MAX || c->heads <= 0 || c->heads > 65535 ||
      c->head_dim <= 0 || c->head_dim % 8 || c->head_dim > KV_DIM_MAX || c->table_pages <= 0 || c->seqs < 0 ||
      (long long)c->table_pages * c->page_size > DIM_MAX)
    return false;
  if (c->seqs == 0) return true;
  if (!c->k || !c->v || !al16(c->k) || !al16(c->v) || !c->k_scale || !c->v_scale || ((uintptr_t)c->k_scale & 3) ||
      ((uintptr_t)c->v_scale & 3) || !c->table || !c->lens || ((uintptr_t)c->table & 3) || ((uintptr_t)c->lens & 3) ||
      (c->seqs > 1 && c->ld_table < c->table_pages))
    return false;
  return strides_ok(*c, c->k_stride, c->head_dim, 16) && strides_ok(*c, c->v_stride, c->head_dim, 16) &&
         strides_ok(*c, c->k_scale_stride, 1, 1) && strides_ok(*c, c->v_scale_stride, 1, 1);
}
featfix_status kv_rows(int dtype, const featfix_kv_cache* cache, const KvRows& r,
                       cudaError_t (*launch)(DType, const KvCache&, const KvRows&, cudaStream_t), void* stream) {
  if (!dt_ok(dtype) || !cache_ok(cache) || r.rows < 0 || r.rows > DIM_MAX) return FEATFIX_ERR_INVALID_ARG;
  if (!r.row_start && r.rows != cache->seqs) return FEATFIX_ERR_INVALID_ARG;
  if (r.rows == 0 || cache->seqs == 0) return FEATFIX_OK;
  const long long width = (long long)cache->heads * cache->head_dim;
  if (!r.k || !r.v || r.ldk < width || r.ldv < width || !el_al(dtype, {r.k, r.v}) || ((uintptr_t)r.row_start & 3))
    return FEATFIX_ERR_INVALID_ARG;
  return st(launch((DType)dtype, *cache, r, (cudaStream_t)stream));
}

}  // namespace

extern "C" {

featfix_status featfix_op_draft(int dtype, void* dev_x, const void* const* dev_hist, const double* w, int n_terms,
                                long long n, void* stream) {
  if (!dt_ok(dtype) || !dev_x || !dev_hist || !w || n_terms < 1 || n_terms > 4 || n < 0) return FEATFIX_ERR_INVALID_ARG;
  Hist4 h = {{nullptr, nullptr, nullptr, nullptr}};
  float wf[4] = {0, 0, 0, 0};
  if (!al16(dev_x)) return FEATFIX_ERR_INVALID_ARG;
  for (int j = 0; j < n_terms; ++j) {
    if (!dev_hist[j] || !al16(dev_hist[j])) return FEATFIX_ERR_INVALID_ARG;
    h.p[j] = dev_hist[j];
    wf[j] = (float)w[j];
  }
  return st(launch_draft((DType)dtype, dev_x, h, wf, n_terms, n, (cudaStream_t)stream));
}

size_t featfix_op_verify_workspace(long long n) { return verify_workspace_bytes(n); }

featfix_status featfix_op_verify(int dtype, void* dev_u, const void* const* dev_hist, const double* w, int n_terms,
                                 const void* dev_hf, long long n, int write_draft, double* dev_sums,
                                 void* dev_workspace, size_t ws_bytes, void* stream) {
  if (!dt_ok(dtype) || !dev_u || !dev_hist || !w || !dev_hf || !dev_sums || !dev_workspace || n_terms < 1 ||
      n_terms > 4 || n <= 0)
    return FEATFIX_ERR_INVALID_ARG;
  if (ws_bytes < verify_workspace_bytes(n)) return FEATFIX_ERR_INVALID_ARG;
  if (!al16(dev_u) || !al16(dev_hf) || !al16(dev_workspace)) return FEATFIX_ERR_INVALID_ARG;
  Hist4 h = {{nullptr, nullptr, nullptr, nullptr}};
  float wf[4] = {0, 0, 0, 0};
  for (int j = 0; j < n_terms; ++j) {
    if (!dev_hist[j] || !al16(dev_hist[j])) return FEATFIX_ERR_INVALID_ARG;
    h.p[j] = dev_hist[j];
    wf[j] = (float)w[j];
  }
  return st(launch_verify((DType)dtype, dev_u, h, wf, n_terms, dev_hf, n, write_draft, dev_sums, dev_workspace,
                          (cudaStream_t)stream));
}

featfix_status featfix_op_ln_modulate(int dtype, const void* dev_x, void* dev_out, long long rows, int C,
                                      const float* dev_shift, const float* dev_scale, int mod_stride,
                                      int rows_per_batch, void* stream) {
  if (!dt_ok(dtype) || !dev_x || !dev_out || !dev_shift || !dev_scale || rows < 0 || C <= 0 || rows_per_batch <= 0)
    return FEATFIX_ERR_INVALID_ARG;
  if (C % (dtype == FEATFIX_DTYPE_F32 ? 4 : 8)) return FEATFIX_ERR_INVALID_ARG;
  return st(launch_ln_mod((DType)dtype, dev_x, dev_out, rows, C, dev_shift, dev_scale, mod_stride, 0, 1,
                          rows_per_batch, (cudaStream_t)stream));
}

featfix_status featfix_op_gemm(int dtype, int M, int N, int K, const void* dev_a, const void* dev_w,
                               const void* dev_bias, int act, const float* dev_gate, int gate_stride,
                               int rows_per_batch, const void* dev_resid, void* dev_out, const void* dev_hist_base,
                               void* dev_hist_out, void* stream) {
  if (!dt_ok(dtype) || M < 0 || N <= 0 || K <= 0 || !dev_a || !dev_w || !dev_out) return FEATFIX_ERR_INVALID_ARG;
  if (act != 0 && act != 1) return FEATFIX_ERR_INVALID_ARG;
  if ((dev_gate != nullptr) && (rows_per_batch <= 0 || gate_stride < N)) return FEATFIX_ERR_INVALID_ARG;
  if ((dev_hist_out != nullptr) != (dev_hist_base != nullptr)) return FEATFIX_ERR_INVALID_ARG;
  if (N % (dtype == FEATFIX_DTYPE_F32 ? 4 : 8)) return FEATFIX_ERR_INVALID_ARG;
  EpiArgs e = epi_plain(dev_out, N);
  e.bias = dev_bias;
  e.act = act;
  e.gate = dev_gate;
  e.gate_stride = gate_stride;
  e.rpb1 = rows_per_batch > 0 ? rows_per_batch : 1;
  e.resid = dev_resid;
  e.ld_resid = N;
  e.hist_base = dev_hist_base;
  e.hist_out = dev_hist_out;
  if (dtype == FEATFIX_DTYPE_BF16) return st(gemm_tc(M, N, K, dev_a, K, dev_w, K, e, (cudaStream_t)stream));
  return st(gemm_f32(M, N, K, (const float*)dev_a, K, (const float*)dev_w, K, e, (cudaStream_t)stream));
}

featfix_status featfix_op_attention(int dtype, const void* dev_qkv, int ld_qkv, void* dev_out, int ld_out, int batch,
                                    int n_txt, int n_img, int heads, int head_dim, void* stream) {
  if (!dt_ok(dtype) || !dev_qkv || !dev_out || batch <= 0 || n_txt < 0 || n_img < 0 || heads <= 0 ||
      head_dim <= 0 || head_dim % 8 || head_dim > 128)
    return FEATFIX_ERR_INVALID_ARG;
  const int C = heads * head_dim;
  if (ld_qkv < 3 * C || ld_out < C) return FEATFIX_ERR_INVALID_ARG;
  const int es = dtype == FEATFIX_DTYPE_F32 ? 4 : 2;
  const char* base = reinterpret_cast<const char*>(dev_qkv);
  AttnArgs a;
  a.q = base;
  a.k = base + (size_t)C * es;
  a.v = base + (size_t)2 * C * es;
  a.ld_qkv = ld_qkv;
  a.out = dev_out;
  a.ld_out = ld_out;
  a.B = batch;
  a.Nt = n_txt;
  a.Ni = n_img;
  a.H = heads;
  a.hd = head_dim;
  return st(attention((DType)dtype, a, (cudaStream_t)stream));
}

featfix_status featfix_op_rms_norm(int dtype, long long rows, int C, const void* dev_x, long long ld_x,
                                   const void* dev_resid, long long ld_resid, void* dev_sum, long long ld_sum,
                                   const void* dev_weight, float eps, void* dev_out, long long ld_out, void* dev_q,
                                   long long ld_q, float* dev_scale, long long ld_scale, void* stream) {
  if (!dt_ok(dtype) || rows < 0 || rows > DIM_MAX || C <= 0 || C > RMS_COLS_MAX || !(eps >= 0.f))
    return FEATFIX_ERR_INVALID_ARG;
  if (rows == 0) return FEATFIX_OK;
  if (!dev_x || ld_x < C || (dev_out != nullptr) == (dev_q != nullptr)) return FEATFIX_ERR_INVALID_ARG;
  if ((dev_resid && ld_resid < C) || (dev_sum && ld_sum < C) || (dev_out && ld_out < C)) return FEATFIX_ERR_INVALID_ARG;
  if (!el_al(dtype, {dev_x, dev_resid, dev_sum, dev_weight, dev_out})) return FEATFIX_ERR_INVALID_ARG;
  const Quant8Out q8 = {dev_q, ld_q, dev_scale, ld_scale};
  if (dev_q && !q8_ok(q8, C, rows)) return FEATFIX_ERR_INVALID_ARG;
  const RmsArgs a = {dev_x, ld_x, dev_resid, ld_resid, dev_sum, ld_sum, dev_weight, eps, dev_out, ld_out, q8};
  return st(launch_rms_norm((DType)dtype, rows, C, a, (cudaStream_t)stream));
}

featfix_status featfix_op_quant8(int dtype, int tile, long long rows, int cols, const void* dev_x, long long ld_x,
                                 void* dev_q, long long ld_q, float* dev_scale, long long ld_scale, void* stream) {
  if (!dt_ok(dtype) || (tile != 1 && tile != 128) || rows < 0 || rows > DIM_MAX || cols <= 0 || cols > DIM_MAX)
    return FEATFIX_ERR_INVALID_ARG;
  if (rows == 0) return FEATFIX_OK;
  if (!dev_x || ld_x < cols) return FEATFIX_ERR_INVALID_ARG;
  const Quant8Out q8 = {dev_q, ld_q, dev_scale, ld_scale};
  if (!el_al(dtype, {dev_x}) || !q8_ok(q8, cols, tile == 1 ? rows : (cols + 127) / 128)) return FEATFIX_ERR_INVALID_ARG;
  return st(launch_quant8((DType)dtype, tile, rows, cols, dev_x, ld_x, q8, (cudaStream_t)stream));
}

featfix_status featfix_op_gemm8(int dtype, int M, int N, int K, const void* dev_a, long long ld_a,
                                const float* dev_a_scale, long long ld_a_scale, const void* dev_w, long long ld_w,
                                const float* dev_w_scale, long long ld_w_scale, const void* dev_bias, int act,
                                const float* dev_gate, long long gate_stride, int rows_per_batch, const void* dev_resid,
                                long long ld_resid, void* dev_out, long long ld_out, void* dev_q, long long ld_q,
                                float* dev_q_scale, long long ld_q_scale, void* stream) {
  if (!dt_ok(dtype) || M < 0 || N <= 0 || K <= 0 || M > DIM_MAX || N > DIM_MAX || K > DIM_MAX || (act != 0 && act != 1))
    return FEATFIX_ERR_INVALID_ARG;
  if (M == 0) return FEATFIX_OK;
  if ((dev_out != nullptr) == (dev_q != nullptr)) return FEATFIX_ERR_INVALID_ARG;
  // (the operands' scales are only read: q8_ok asks for the same of inputs and outputs)
  const Quant8Out a8 = {const_cast<void*>(dev_a), ld_a, const_cast<float*>(dev_a_scale), ld_a_scale};
  const Quant8Out w8 = {const_cast<void*>(dev_w), ld_w, const_cast<float*>(dev_w_scale), ld_w_scale};
  const Quant8Out q8 = {dev_q, ld_q, dev_q_scale, ld_q_scale};
  if (!q8_ok(a8, K, M) || !q8_ok(w8, K, ((long long)K + 127) / 128) || (dev_q && !q8_ok(q8, N, M)))
    return FEATFIX_ERR_INVALID_ARG;
  if (dev_q && (dev_gate || dev_resid)) return FEATFIX_ERR_INVALID_ARG;
  if (dev_gate && (rows_per_batch <= 0 || gate_stride < N || ((uintptr_t)dev_gate & 3))) return FEATFIX_ERR_INVALID_ARG;
  if ((dev_resid && ld_resid < N) || (dev_out && ld_out < N) || !el_al(dtype, {dev_bias, dev_resid, dev_out}))
    return FEATFIX_ERR_INVALID_ARG;
  const Gemm8Args g = {dev_a, ld_a, dev_a_scale, ld_a_scale, dev_w, ld_w, dev_w_scale, ld_w_scale, dev_bias, act,
                       dev_gate, gate_stride, rows_per_batch > 0 ? rows_per_batch : 1, dev_resid, ld_resid, dev_out,
                       ld_out, q8};
  return st(gemm8((DType)dtype, M, N, K, g, (cudaStream_t)stream));
}

featfix_status featfix_op_gemm8_watchdog(void) {
  unsigned int flags = 0;
  return gemm8_watchdog_take(&flags) == cudaSuccess && !flags ? FEATFIX_OK : FEATFIX_ERR_CUDA;
}

featfix_status featfix_op_gemm8_watchdog_probe(unsigned long long* limit_ns) {
  unsigned long long t[2] = {0, 0};
  const cudaError_t e = gemm8_watchdog_probe(t);
  if (limit_ns)
    for (int i = 0; i < 2; ++i) limit_ns[i] = t[i];
  return st(e);
}

featfix_status featfix_op_rope(int dtype, long long rows, int head_dim, int n_axes, const int* axis_dims,
                               const int* dev_pos, long long ld_pos, double theta, unsigned flags, const void* dev_q,
                               long long ld_q, int q_heads, const void* dev_q_weight, void* dev_q_out,
                               long long ld_q_out, const void* dev_k, long long ld_k, int k_heads,
                               const void* dev_k_weight, void* dev_k_out, long long ld_k_out, float eps,
                               void* stream) {
  if (!dt_ok(dtype) || rows < 0 || rows > DIM_MAX || head_dim <= 0 || head_dim % 2 || head_dim > 2 * ROPE_PAIRS ||
      n_axes < 1 || n_axes > 8 || !axis_dims ||
      !(theta > 0.0) || isinf(theta) || (flags & ~7u) || q_heads < 0 || k_heads < 0 || q_heads + (long long)k_heads < 1 ||
      q_heads + (long long)k_heads > 65535 ||
      !(eps >= 0.f))
    return FEATFIX_ERR_INVALID_ARG;
  int rot = 0;
  for (int a = 0; a < n_axes; ++a) {
    if (axis_dims[a] <= 0 || axis_dims[a] % 2 || axis_dims[a] > head_dim - rot) return FEATFIX_ERR_INVALID_ARG;
    rot += axis_dims[a];
  }
  if (rows == 0) return FEATFIX_OK;
  if (!dev_pos || ((uintptr_t)dev_pos & 3) || ld_pos < rows) return FEATFIX_ERR_INVALID_ARG;
  RopeArgs r = {};
  r.side[0] = {dev_q, ld_q, dev_q_out, ld_q_out, dev_q_weight, q_heads};
  r.side[1] = {dev_k, ld_k, dev_k_out, ld_k_out, dev_k_weight, k_heads};
  for (const RopeSide& sd : r.side) {
    const long long width = (long long)sd.heads * head_dim;
    if (sd.heads == 0) continue;
    if (!sd.x || !sd.out || width > 0x7fffffff || sd.ldx < width || sd.ldo < width ||
        !el_al(dtype, {sd.x, sd.out, sd.weight}) || (sd.weight && (flags & FEATFIX_ROPE_INVERSE)))
      return FEATFIX_ERR_INVALID_ARG;
  }
  r.pos = dev_pos;
  r.ld_pos = ld_pos;
  r.hd = head_dim;
  r.rot = rot;
  r.halves = (flags & FEATFIX_ROPE_HALVES) ? 1 : 0;
  r.eps = eps;
  // turns per position: theta^(-2 i / width) / 2 pi, each step of a ladder one product
  const double turn = ((flags & FEATFIX_ROPE_INVERSE) ? -0.5 : 0.5) / M_PI;
  const bool one = (flags & FEATFIX_ROPE_ONE_LADDER) != 0;
  double f = turn, step = one ? pow(theta, -2.0 / rot) : 1.0;
  for (int a = 0, p = 0; a < n_axes; ++a) {
    if (!one) {
      f = turn;
      step = pow(theta, -2.0 / axis_dims[a]);
    }
    for (int i = 0; i < axis_dims[a] / 2; ++i, ++p, f *= step) {
      const float hi = (float)f;
      r.freq[p] = make_float2(hi, (float)(f - (double)hi));
      r.axis[p] = (unsigned char)a;
    }
  }
  return st(launch_rope((DType)dtype, rows, r, (cudaStream_t)stream));
}

featfix_status featfix_op_kv_write(int dtype, const featfix_kv_cache* cache, long long rows, const int* dev_row_start,
                                   const void* dev_k, long long ld_k, const void* dev_v, long long ld_v, void* stream) {
  // (k and v are only read)
  return kv_rows(dtype, cache, {rows, dev_row_start, const_cast<void*>(dev_k), ld_k, const_cast<void*>(dev_v), ld_v},
                 launch_kv_write, stream);
}

featfix_status featfix_op_kv_read(int dtype, const featfix_kv_cache* cache, long long rows, const int* dev_row_start,
                                  void* dev_k, long long ld_k, void* dev_v, long long ld_v, void* stream) {
  return kv_rows(dtype, cache, {rows, dev_row_start, dev_k, ld_k, dev_v, ld_v}, launch_kv_read, stream);
}

size_t featfix_op_kv_attention_workspace(int seqs, int q_heads, int k_heads, int head_dim, long long tokens) {
  if (seqs <= 0 || q_heads <= 0 || q_heads > 65535 || k_heads <= 0 || q_heads % k_heads || head_dim <= 0 ||
      head_dim % 8 || head_dim > KV_DIM_MAX || tokens <= 0 || tokens > DIM_MAX)
    return 0;
  return kv_attention_workspace(seqs, q_heads, k_heads, head_dim, tokens);
}

featfix_status featfix_op_kv_attention(int dtype, const featfix_kv_cache* cache, const void* dev_q, long long ld_q,
                                       int q_heads, float scale, int window, void* dev_out, long long ld_out,
                                       float* dev_lse, void* dev_workspace, size_t ws_bytes, void* stream) {
  if (!dt_ok(dtype) || !cache_ok(cache) || q_heads <= 0 || q_heads > 65535 || q_heads % cache->heads || window < 0 ||
      !isfinite(scale))
    return FEATFIX_ERR_INVALID_ARG;
  if (cache->seqs == 0) return FEATFIX_OK;
  const long long width = (long long)q_heads * cache->head_dim;
  if (!dev_q || !dev_out || ld_q < width || ld_out < width || !el_al(dtype, {dev_q, dev_out}) || ((uintptr_t)dev_lse & 3))
    return FEATFIX_ERR_INVALID_ARG;
  const size_t need = kv_attention_workspace(cache->seqs, q_heads, cache->heads, cache->head_dim,
                                             (long long)cache->table_pages * cache->page_size);
  if (need && (!dev_workspace || ws_bytes < need || !al16(dev_workspace))) return FEATFIX_ERR_INVALID_ARG;
  const KvAttnArgs a = {dev_q, ld_q, dev_out, ld_out, dev_lse, q_heads, scale, window, dev_workspace};
  return st(launch_kv_attention((DType)dtype, *cache, a, (cudaStream_t)stream));
}

featfix_status featfix_op_block_norms(int dtype, long long rows, int C, unsigned flags, float eps, const void* dev_y,
                                      long long ld_y, const void* dev_weight_after, const float* dev_gate,
                                      long long gate_stride, const void* dev_x, long long ld_x, float resid_scale,
                                      void* dev_sum, long long ld_sum, const void* dev_weight, const float* dev_scale,
                                      long long scale_stride, const float* dev_shift, long long shift_stride,
                                      int rows_per_batch, void* dev_out, long long ld_out, void* dev_q, long long ld_q,
                                      float* dev_q_scale, long long ld_q_scale, void* stream) {
  if (!dt_ok(dtype) || rows < 0 || rows > DIM_MAX || C <= 0 || C > BLOCK_NORMS_COLS_MAX || !(eps >= 0.f) || (flags & ~3u) ||
      !isfinite(resid_scale))
    return FEATFIX_ERR_INVALID_ARG;
  if (rows == 0) return FEATFIX_OK;
  if (!dev_y || ld_y < C || (dev_out && dev_q) || (!dev_sum && !dev_out && !dev_q) ||
      (dev_weight_after && !(flags & FEATFIX_NORM_AFTER)))
    return FEATFIX_ERR_INVALID_ARG;
  if ((dev_x && ld_x < C) || (dev_sum && ld_sum < C) || (dev_out && ld_out < C)) return FEATFIX_ERR_INVALID_ARG;
  if (!el_al(dtype, {dev_y, dev_weight_after, dev_x, dev_sum, dev_weight, dev_out}) ||
      (((uintptr_t)dev_gate | (uintptr_t)dev_scale | (uintptr_t)dev_shift) & 3))
    return FEATFIX_ERR_INVALID_ARG;
  if ((dev_gate || dev_scale || dev_shift) && rows_per_batch <= 0) return FEATFIX_ERR_INVALID_ARG;
  // (one sample has no stride)
  const bool many = rows > rows_per_batch;
  if (many && ((dev_gate && gate_stride < C) || (dev_scale && scale_stride < C) || (dev_shift && shift_stride < C)))
    return FEATFIX_ERR_INVALID_ARG;
  const Quant8Out q8 = {dev_q, ld_q, dev_q_scale, ld_q_scale};
  if (dev_q && !q8_ok(q8, C, rows)) return FEATFIX_ERR_INVALID_ARG;
  const BlockNormsArgs a = {dev_y, ld_y, dev_weight_after, dev_gate, gate_stride, dev_x, ld_x, resid_scale, dev_sum,
                            ld_sum, dev_weight, dev_scale, scale_stride, dev_shift, shift_stride,
                            rows_per_batch > 0 ? rows_per_batch : 1, (flags & FEATFIX_NORM_AFTER) != 0,
                            (flags & FEATFIX_NORM_CENTERED) != 0, eps, dev_out, ld_out, q8};
  return st(launch_block_norms((DType)dtype, rows, C, a, (cudaStream_t)stream));
}

}  // extern "C"
