/*
 * featfix_ops.h -- the individual kernels of the FeatFix hot path, exposed on
 * caller buffers so each can be tested and timed on its own.  The context
 * API in featfix.h composes exactly these kernels.
 *
 * Common rules: dev_* pointers are device memory on the current device and
 * stay owned by the caller; `stream` is a cudaStream_t (NULL = legacy
 * default stream); dtype is FEATFIX_DTYPE_F32 or FEATFIX_DTYPE_BF16; every
 * pointer must be 16-byte aligned and every element count that is read with
 * 16-byte vectors must keep that alignment (row strides in elements a
 * multiple of 8 for bf16, 4 for f32).  Work is enqueued asynchronously;
 * launch-configuration errors return FEATFIX_ERR_CUDA, argument errors
 * FEATFIX_ERR_INVALID_ARG, and nothing aborts or traps.
 */
#ifndef FEATFIX_OPS_H
#define FEATFIX_OPS_H

#include <stddef.h>
#include "featfix.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Draft of Eq. 2 in weight form: x[i] <- x[i] + sum_{j<n_terms} w[j]*hist[j][i]
 * for i < n.  hist[j] is the increment h^f - u stored at the j-th newest
 * refresh; w are the Taylor/Lagrange weights of featfix_plan_build
 * (n_terms = K_eff + 1 <= 4).  Arithmetic in fp32, result rounded to dtype.
 * In place on dev_x.                                                        */
FEATFIX_API featfix_status featfix_op_draft(int dtype, void* dev_x, const void* const* dev_hist, const double* w,
                                int n_terms, long long n, void* stream);

/* Scratch bytes featfix_op_verify needs for n elements.                    */
FEATFIX_API size_t featfix_op_verify_workspace(long long n);

/* Paid check at a site (Eqs. 3-5): forms h_d = u + sum_j w[j]*hist[j]
 * elementwise from the same incoming state dev_u, compares it with the exact
 * output dev_hf and writes the four sums
 *   dev_sums[0] = sum |h_d - h_f|,  dev_sums[1] = sum |h_f|,
 *   dev_sums[2] = sum (h_d - h_f)^2, dev_sums[3] = sum h_f^2
 * (double, device) with a fixed, run-to-run deterministic reduction order.
 * write_draft != 0 (Verify arm) also overwrites dev_u with h_d.  The per-CTA
 * partial sums live in dev_workspace (>= featfix_op_verify_workspace(n)
 * bytes, caller-owned).                                                     */
FEATFIX_API featfix_status featfix_op_verify(int dtype, void* dev_u, const void* const* dev_hist, const double* w,
                                 int n_terms, const void* dev_hf, long long n, int write_draft,
                                 double* dev_sums, void* dev_workspace, size_t ws_bytes, void* stream);

/* featfix_op_verify without any device allocation.  The paper has no
 * counterpart: this is a deployment convenience.
 *
 * Some callers cannot allocate device memory at all: a host application or
 * plugin framework that owns every byte of the GPU and forbids side
 * allocations, a memory-budgeted service that plans all device memory up
 * front, or a latency-critical loop where a cudaMalloc (with its implicit
 * synchronisation and possible failure) is not acceptable.  For them this
 * entry point computes exactly what featfix_op_verify computes (same sums,
 * same deterministic reduction order, same Verify-arm write of h_d) with the
 * per-cluster partial sums kept in a fixed scratch array of
 * FEATFIX_VERIFY_NOALLOC_SCRATCH_BYTES (16 KiB) compiled into the library.
 * The caller still provides dev_u, dev_hist, dev_hf and dev_sums.
 *
 *  - No cudaMalloc, cudaFree or other allocating routine is called.  Every
 *    GPU that loads the library holds the 16 KiB array until the process
 *    exits.
 *  - Every call looks up the array's device address with the calling
 *    thread's current device; the first call on a device may load the
 *    library's module there, so make that first call before any stream
 *    capture on the device.
 *  - A call needs featfix_op_verify_workspace(n) bytes of the array (one
 *    32-byte partial per 8-CTA cluster, at most 4 CTAs per SM); if that is
 *    more than 16 KiB (a GPU with more than 1024 SMs) the call returns
 *    FEATFIX_ERR_INVALID_ARG and launches nothing.
 *  - All calls, on every stream of a device, share the one array, which
 *    keeps the last call's contents.  Each launch writes every partial it
 *    reads back, so nothing needs clearing; but calls whose executions
 *    overlap on the GPU race on the array and may return wrong sums:
 *    serialise them (one stream, or events between streams).             */
#define FEATFIX_VERIFY_NOALLOC_SCRATCH_BYTES 16384
FEATFIX_API featfix_status featfix_op_verify_noalloc(int dtype, void* dev_u, const void* const* dev_hist,
                                                     const double* w, int n_terms, const void* dev_hf, long long n,
                                                     int write_draft, double* dev_sums, void* stream);

/* adaLN input of a branch: out[r,:] = LN(x[r,:]) * (1 + scale[b,:]) + shift[b,:]
 * with LN over C columns without affine (eps 1e-6), b = r / rows_per_batch,
 * shift/scale float32 rows of stride mod_stride.  x, out row-major [rows, C]. */
FEATFIX_API featfix_status featfix_op_ln_modulate(int dtype, const void* dev_x, void* dev_out, long long rows, int C,
                                      const float* dev_shift, const float* dev_scale, int mod_stride,
                                      int rows_per_batch, void* stream);

/* Linear layer with the block's fused epilogue:
 *   y = act(A W^T + bias);  out = resid + gate[b,:] * y  (or out = y)
 *   hist_out = out - hist_base                              (optional)
 * A [M,K] row-major (lda = K), W [N,K] (nn.Linear weight), bias [N] in
 * dtype; act 0 = identity, 1 = GELU (tanh); gate float32 rows of stride
 * gate_stride picked by b = row / rows_per_batch (NULL = no gate/resid);
 * resid, out, hist_base, hist_out [M,N] dtype with row stride N.  bf16 runs on
 * tcgen05 tensor cores with TMEM accumulators fed by TMA (K % 8 == 0);
 * f32 runs a CUDA-core kernel without TF32.                               */
FEATFIX_API featfix_status featfix_op_gemm(int dtype, int M, int N, int K, const void* dev_a, const void* dev_w,
                               const void* dev_bias, int act, const float* dev_gate, int gate_stride,
                               int rows_per_batch, const void* dev_resid, void* dev_out,
                               const void* dev_hist_base, void* dev_hist_out, void* stream);

/* Non-causal multi-head attention softmax(q k^T / sqrt(d)) v over the joint
 * [text ; image] sequence of each sample.  dev_qkv holds, for every token row
 * (featfix_token_row layout with batch samples, n_txt text and n_img image
 * tokens), q | k | v of H heads of width d at columns [0,C), [C,2C), [2C,3C),
 * row stride ld_qkv elements.  dev_out receives o [rows, C] with row stride
 * ld_out.  d % 8 == 0 and d <= 128.                                        */
FEATFIX_API featfix_status featfix_op_attention(int dtype, const void* dev_qkv, int ld_qkv, void* dev_out, int ld_out,
                                    int batch, int n_txt, int n_img, int heads, int head_dim,
                                    void* stream);

/* ---------------------------------------------------------------------------
 * 8-bit transformer layers: a root-mean-square norm, a product and a
 * quantiser on e4m3 values with a scale for each block of 128 along the
 * reduction dimension, and rotary positions with several axes.  They serve
 * pre-norm transformer layers beside the denoiser's own adaLN blocks; the paper
 * has no counterpart.
 *
 * 8-bit tensors are e4m3 bytes (largest value 448), row-major with a row stride
 * ld of at least the width and a multiple of 16.  A block's scale is
 *   s = max(largest |x| of the block / 448, 2^-100),   q = e4m3(x / s)
 * rounded to nearest even (both within a few 2^-24: a quotient that near a tie may take
 * either code); a block stands for q * s.  A NaN in a block makes its
 * scale NaN, an infinity makes it infinite: what is computed from the block is
 * NaN, never a finite number.  Activations have one scale per row and 128
 * columns, stored block by block: the scale of row r and column c is
 * scale[(c / 128) * ld_scale + r], ld_scale >= rows.  Weights have one per
 * 128 x 128 block: scale[(r / 128) * ld_scale + c / 128],
 * ld_scale >= ceil(cols / 128).
 *
 * Pointers to 8-bit tensors are 16-byte aligned, all others need only their
 * element's alignment (16-byte aligned rows are faster); dtypes are
 * FEATFIX_DTYPE_F32 / _BF16; row strides are in elements.  Sizes of zero rows
 * are allowed and do nothing; no dimension exceeds 2^31 - 256.  No call allocates or
 * keeps anything.
 * ------------------------------------------------------------------------- */

/* Root-mean-square norm of rows of C columns (C <= 32768) with the residual's
 * addition in front of it:
 *   h = x + resid   (x alone where dev_resid is NULL),
 *   y = h / sqrt(mean(h^2) + eps) * weight   (weight 1 where dev_weight is NULL).
 * h and its sum of squares are kept in fp32 (rows whose sum passes fp32's range, |h| of
 * about 1e19, have y = 0); dev_sum (NULL: not wanted) receives it rounded
 * to dtype and may be dev_x or dev_resid.  Exactly one of dev_out (y in dtype)
 * and dev_q (y in 8 bits, with dev_scale) is given.                          */
FEATFIX_API featfix_status featfix_op_rms_norm(int dtype, long long rows, int C, const void* dev_x, long long ld_x,
                                   const void* dev_resid, long long ld_resid, void* dev_sum, long long ld_sum,
                                   const void* dev_weight, float eps, void* dev_out, long long ld_out, void* dev_q,
                                   long long ld_q, float* dev_scale, long long ld_scale, void* stream);

/* x [rows, cols] in 8 bits: tile 1 for activations, 128 for weights (the
 * scales' layouts above).                                                    */
FEATFIX_API featfix_status featfix_op_quant8(int dtype, int tile, long long rows, int cols, const void* dev_x,
                                 long long ld_x, void* dev_q, long long ld_q, float* dev_scale, long long ld_scale,
                                 void* stream);

/* Linear layer on 8-bit activations A [M, K] and weights W [N, K]:
 *   acc[m, n] = sum_b a_scale[b, m] w_scale[n / 128, b] sum_{k in block b} A[m, k] W[n, k],
 *   y = act(acc + bias),   act 0 = identity, 1 = GELU (tanh),
 * with fp32 accumulation.  Exactly one of the results is given:
 *   dev_out: resid + gate[m / rows_per_batch, :] * y in dtype [M, N] (gate float
 *            rows of stride gate_stride, without it y; resid in dtype; both
 *            nullable);
 *   dev_q:   y in 8 bits with dev_q_scale, for the next layer (no gate, no resid).
 * bias [N] is in dtype.  dev_out may be dev_resid where both have one row stride.
 * A scale product a_scale * w_scale past fp32's range makes the result infinite
 * or zero.  tcgen05 tensor cores (kind::f8f6f4), fed by TMA.                 */
FEATFIX_API featfix_status featfix_op_gemm8(int dtype, int M, int N, int K, const void* dev_a, long long ld_a,
                                const float* dev_a_scale, long long ld_a_scale, const void* dev_w, long long ld_w,
                                const float* dev_w_scale, long long ld_w_scale, const void* dev_bias, int act,
                                const float* dev_gate, long long gate_stride, int rows_per_batch, const void* dev_resid,
                                long long ld_resid, void* dev_out, long long ld_out, void* dev_q, long long ld_q,
                                float* dev_q_scale, long long ld_q_scale, void* stream);

/* Waits for the current device and returns FEATFIX_ERR_CUDA if a bounded wait inside a
 * featfix_op_gemm8 kernel gave up since the last call (its results are then
 * incomplete), FEATFIX_OK otherwise.  Nothing else reports it: a program asks at its own
 * checkpoints.  Not for use while a stream is captured.                        */
FEATFIX_API featfix_status featfix_op_gemm8_watchdog(void);

/* Failure-detection test hook.  Lets the two bounded waits of featfix_op_gemm8's kernels
 * run out on the current device, on barriers that nothing arrives on, after a 32nd of
 * their limits (0.13 s): they raise the flag that featfix_op_gemm8_watchdog reports, the
 * kernel returns, nothing traps.  limit_ns[2] (host, nullable) receives the limits, 32
 * times what the waits took.  Uses the default stream and waits for it.        */
FEATFIX_API featfix_status featfix_op_gemm8_watchdog_probe(unsigned long long* limit_ns);

/* Rotary positions on the heads of q [rows, q_heads * head_dim] and k [rows,
 * k_heads * head_dim] (shared key heads: k_heads below q_heads; either may be
 * absent with 0 heads).  axis_dims (host, n_axes even numbers, n_axes <= 8) are the
 * widths of a head that each axis turns, one after the other; their sum rot <=
 * head_dim, the columns past it are only copied.  Pair p, the i-th of axis a, of
 * row r turns by
 *   pos[a * ld_pos + r] * theta^(-2 i / axis_dims[a]),
 * or theta^(-2 p / rot) with FEATFIX_ROPE_ONE_LADDER; with theta >= 1 the angle is
 * within fp32 rounding of a turn up to positions of 2^20, and within 3e-5 at any
 * int32.  Pairs are columns (2p, 2p + 1), or (p, p + rot / 2) with
 * FEATFIX_ROPE_HALVES.  FEATFIX_ROPE_INVERSE turns the other way: the inverse and
 * so the gradient of the rotation.  q_weight / k_weight ([head_dim] in dtype,
 * nullable) put the root-mean-square norm of each head, times the weight, in front
 * of the rotation (not with INVERSE).  Outputs may be their inputs.  head_dim is
 * even and at most 256, q_heads + k_heads at most 65535.                                                      */
#define FEATFIX_ROPE_HALVES 1u
#define FEATFIX_ROPE_ONE_LADDER 2u
#define FEATFIX_ROPE_INVERSE 4u
FEATFIX_API featfix_status featfix_op_rope(int dtype, long long rows, int head_dim, int n_axes, const int* axis_dims,
                               const int* dev_pos, long long ld_pos, double theta, unsigned flags, const void* dev_q,
                               long long ld_q, int q_heads, const void* dev_q_weight, void* dev_q_out,
                               long long ld_q_out, const void* dev_k, long long ld_k, int k_heads,
                               const void* dev_k_weight, void* dev_k_out, long long ld_k_out, float eps,
                               void* stream);

/* ---------------------------------------------------------------------------
 * An 8-bit cache of keys and values in pages, and the attention of one new token
 * of each sequence over it.  A program that makes tokens one after another, or a
 * clip piece by piece, keeps what later tokens attend to in it.  Several new tokens of
 * one sequence attend as several sequences, with the same pages and each token's own
 * length; every one of them reads the cache.  (The paper has no counterpart.)
 *
 * A place of the cache holds a head of one token: head_dim e4m3 values and one
 * scale, by the rule above with the head as the block:
 *   s = max(largest |x| of the head / 448, 2^-100),   q = e4m3(x / s).
 * Scales that are NaN, infinite or negative stand for NaN in all of the head.
 *
 * k, v are e4m3 bytes; place (page, slot, head) starts stride[0] * page +
 * stride[1] * slot + stride[2] * head bytes behind the pointer (multiples of 16, at
 * least head_dim; pointers are 16-byte aligned), its scale that many floats behind
 * k_scale / v_scale (at least 1), strides below 2^32: heads inside or outside of a
 * page's tokens, with or without gaps.  head_dim is a multiple of 8, at most 256.
 *
 * Token t of sequence b is in page table[b * ld_table + t / page_size] (t <
 * table_pages * page_size, at most 2^31 - 256), slot t % page_size, for t < lens[b]; lens count the
 * tokens of a call that writes them too.  table and lens are read on the device: a
 * graph that was captured once follows them.  Lengths below 0 count as 0, past the
 * table's end as its end.  A page outside of 0 .. pages - 1 is none: nothing is
 * written to it, its tokens read as zeros and are masked in the attention.  Table
 * places behind a sequence's last token are never looked at, nor are places of the cache.
 * Sequences may share pages that are only read; a page that a call writes to has one
 * place in the table.                                                         */
typedef struct featfix_kv_cache {
  void* k;
  void* v;
  float* k_scale;
  float* v_scale;
  long long k_stride[3], v_stride[3];               /* page, slot, head; bytes  */
  long long k_scale_stride[3], v_scale_stride[3];   /* page, slot, head; floats */
  int pages, page_size, heads, head_dim;
  const int* table;       /* device, [seqs, table_pages], row stride ld_table   */
  long long ld_table;
  int table_pages, seqs;
  const int* lens;        /* device, [seqs]                                     */
} featfix_kv_cache;

/* New tokens into the cache: row dev_row_start[b] + i of k and v [rows, heads *
 * head_dim] becomes token lens[b] - n_b + i of sequence b, n_b = dev_row_start[b + 1] -
 * dev_row_start[b] (device, seqs + 1 rising numbers; NULL: one row to a sequence, rows =
 * seqs).  Rows of no sequence and tokens before the first are skipped.          */
FEATFIX_API featfix_status featfix_op_kv_write(int dtype, const featfix_kv_cache* cache, long long rows,
                                   const int* dev_row_start, const void* dev_k, long long ld_k, const void* dev_v,
                                   long long ld_v, void* stream);

/* The same tokens back, in dtype: the inverse of featfix_op_kv_write.  Tokens before the
 * first are zeros; rows of no sequence are left as they are.                   */
FEATFIX_API featfix_status featfix_op_kv_read(int dtype, const featfix_kv_cache* cache, long long rows,
                                  const int* dev_row_start, void* dev_k, long long ld_k, void* dev_v, long long ld_v,
                                  void* stream);

/* Scratch bytes that featfix_op_kv_attention needs for up to `seqs` sequences in caches of up to
 * `tokens` tokens to each (table_pages * page_size), on any GPU; 0 where it needs none, and for
 * arguments that the operator refuses. */
FEATFIX_API size_t featfix_op_kv_attention_workspace(int seqs, int q_heads, int k_heads, int head_dim,
                                         long long tokens);

/* One new token of each sequence over its cached tokens (itself among them, where it
 * has been written): with t from max(0, lens[b] - window) (window 0: from 0) to lens[b] - 1
 * and h = j / (q_heads / heads),
 *   x_t = scale * q[b, j] . k_t[h],   out[b, j] = sum_t exp(x_t) v_t[h] / sum_t exp(x_t),
 *   lse[b, j] = log sum_t exp(x_t)
 * for the heads j of q [seqs, q_heads * head_dim], q_heads a multiple of the cache's heads;
 * out as q (and may be q, with its row stride), dev_lse [seqs, q_heads] nullable.  A row without
 * tokens has out 0 and lse -infinity.  Scores, sums and statistics are fp32.  q (f32) and weights
 * exp(x_t) v_scale (both dtypes) enter the products as two fp16 terms with a power of two
 * apart: off by 2^-22 of themselves, four times fp32's rounding and far below bf16's, or by
 * 2^-39 of the head's largest, whichever is more; q in bf16 as one, off by the latter alone.
 * Weights below 2^-126 of the largest exp(x_t) are 0.  Results are finite for finite q, k and v
 * with |scale| and head_dim |scale| max|q| max|k| below 2^126.  The workspace (16-byte aligned) may
 * hold anything; calls that may run at the same time need one each.  The same inputs
 * give the same bits.  The largest power of two that divides the page's and the slot's stride
 * times 2^32 must pass the last place's offset (FEATFIX_ERR_UNSUPPORTED: pools from 64 GB on,
 * of places 16 bytes off any rounder stride).                                 */
FEATFIX_API featfix_status featfix_op_kv_attention(int dtype, const featfix_kv_cache* cache, const void* dev_q,
                                       long long ld_q, int q_heads, float scale, int window, void* dev_out,
                                       long long ld_out, float* dev_lse, void* dev_workspace, size_t ws_bytes,
                                       void* stream);

/* The norms at the end of a block and at the beginning of the next one, with the gate and the
 * residual between them, on rows of C columns (C <= 16384), sample s = row / rows_per_batch:
 *   h = resid_scale * x + gate[s] * y'      (x absent: gate[s] * y'),
 *   y' = norm(y) * weight_after with FEATFIX_NORM_AFTER, y without;
 *   z = norm(h) * weight * (1 + scale[s]) + shift[s],
 *   norm(u) = u / sqrt(mean(u^2) + eps), of u - mean(u) with FEATFIX_NORM_CENTERED.
 * Weights [C] in dtype (NULL: 1), gate, scale (NULL: 1 and 0) and shift (NULL: 0) float rows
 * of their strides.  h and all statistics stay in fp32 (rows whose sum of squares passes fp32's
 * range, |u| of about 1e19, have norm 0); dev_sum (nullable) receives h
 * rounded to dtype, dev_out z, or dev_q and dev_q_scale z in 8 bits (scales as activations
 * have them); not both, and at least one of dev_sum, dev_out and dev_q is given.  Outputs may be
 * x or y where they have one row stride.                                        */
#define FEATFIX_NORM_AFTER 1u
#define FEATFIX_NORM_CENTERED 2u
FEATFIX_API featfix_status featfix_op_block_norms(int dtype, long long rows, int C, unsigned flags, float eps,
                                      const void* dev_y, long long ld_y, const void* dev_weight_after,
                                      const float* dev_gate, long long gate_stride, const void* dev_x, long long ld_x,
                                      float resid_scale, void* dev_sum, long long ld_sum, const void* dev_weight,
                                      const float* dev_scale, long long scale_stride, const float* dev_shift,
                                      long long shift_stride, int rows_per_batch, void* dev_out, long long ld_out,
                                      void* dev_q, long long ld_q, float* dev_q_scale, long long ld_q_scale,
                                      void* stream);

#ifdef __cplusplus
}
#endif
#endif /* FEATFIX_OPS_H */
