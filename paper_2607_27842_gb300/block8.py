"""A pre-norm transformer block in 8 bits over the joint [text ; image] rows,
built from the operators of include/featfix_ops.h as a program uses them:

    a      = rms_norm(x) in 8 bits                       featfix_op_rms_norm
    qkv    = a Wqkv^T + b                                featfix_op_gemm8
    q, k   = rotary positions on rms_norm(q), rms_norm(k)  featfix_op_rope
    o      = attention over each sample's rows           featfix_op_attention
    d      = o (in 8 bits) Wproj^T + b                   featfix_op_quant8, featfix_op_gemm8
    x      = x + d;  a = rms_norm(x) in 8 bits           featfix_op_rms_norm
    h      = GELU(a W1^T + b) in 8 bits                  featfix_op_gemm8
    x      = x + h W2^T + b                              featfix_op_gemm8

A plain block: full attention over each sample's rows, as many key heads as query
heads, a GELU MLP; nothing causal, no key cache, no gated activation.  (The
denoiser's own adaLN blocks run inside the library, in bf16 or fp32.)
Rows lie as featfix_token_row has them: the text rows of all samples, then
their image rows.  Every call is asynchronous on the current stream; nothing is
allocated after construction.
"""

import torch

from . import featfix as ff

MATRICES = ("qkv", "proj", "fc1", "fc2")


def joint_positions(batch, n_txt, frames, height, width, device="cuda"):
    """int32 [3, rows]: text token n at (n, 0, 0), the image token of frame f, row
    y and column x at (n_txt + f, y, x), in the row order of featfix_token_row."""
    txt = torch.zeros((batch * n_txt, 3), dtype=torch.int32)
    txt[:, 0] = torch.arange(n_txt, dtype=torch.int32).repeat(batch)
    grid = torch.stack(torch.meshgrid(torch.arange(frames) + n_txt, torch.arange(height), torch.arange(width),
                                      indexing="ij"), -1).reshape(-1, 3).to(torch.int32)
    return torch.cat([txt, grid.repeat(batch, 1)]).t().contiguous().to(device)


def quantized(w):
    """A weight [N, K] (bf16 or fp32, on the GPU) in 8 bits and its scales, as
    featfix_op_gemm8 takes them."""
    n, k = w.shape
    q = torch.zeros((n, (k + 15) // 16 * 16), dtype=torch.uint8, device=w.device)[:, :k]
    scale = torch.empty(((n + 127) // 128, (k + 127) // 128), dtype=torch.float32, device=w.device)
    ff.featfix_op_quant8("f32" if w.dtype == torch.float32 else "bf16", w, q, scale, tile=128)
    return q, scale


class Block8:
    """One block.  ``weights``: bf16 GPU tensors norm1 [C], qkv.w [3C, C], qkv.b,
    q_norm [d], k_norm [d], proj.w [C, C], proj.b, norm2 [C], fc1.w [M, C], fc1.b,
    fc2.w [C, M], fc2.b; the matrices are quantised here, once.  ``axes``: the
    widths of a head that each position axis turns."""

    def __init__(self, weights, heads, axes, batch, n_txt, n_img, theta=10000.0, eps=1e-6):
        self.w = {k: v for k, v in weights.items() if k.removesuffix(".w") not in MATRICES}
        self.q8 = {m: quantized(weights[m + ".w"]) for m in MATRICES}
        self.heads, self.axes, self.theta, self.eps = heads, tuple(axes), theta, eps
        self.batch, self.n_txt, self.n_img = batch, n_txt, n_img
        C, M = weights["fc2.w"].shape
        self.rows, self.C, self.dim = batch * (n_txt + n_img), C, C // heads
        dev = weights["norm1"].device
        self.qkv = torch.empty((self.rows, 3 * C), dtype=torch.bfloat16, device=dev)
        self.o, self.d = (torch.empty((self.rows, C), dtype=torch.bfloat16, device=dev) for _ in range(2))
        # 8-bit activations of width C and M with their scales
        self.a, self.h = ((torch.zeros((self.rows, (n + 15) // 16 * 16), dtype=torch.uint8, device=dev)[:, :n],
                           torch.empty(((n + 127) // 128, self.rows), dtype=torch.float32, device=dev)) for n in (C, M))

    def _linear(self, name, x, **kw):
        ff.featfix_op_gemm8("bf16", *x, *self.q8[name], bias=self.w[name + ".b"], **kw)

    def __call__(self, x, pos):
        """The residual stream x (bf16 [rows, C]) is updated in place; pos int32
        [axes, rows]."""
        C, w = self.C, self.w
        ff.featfix_op_rms_norm("bf16", x, w["norm1"], self.eps, q=self.a[0], q_scale=self.a[1])
        self._linear("qkv", self.a, out=self.qkv)
        q, k = self.qkv[:, :C], self.qkv[:, C:2 * C]
        ff.featfix_op_rope("bf16", pos, self.axes, self.dim, q=q, q_out=q, k=k, k_out=k, theta=self.theta,
                           q_weight=w["q_norm"], k_weight=w["k_norm"], eps=self.eps)
        ff.featfix_op_attention("bf16", self.qkv, self.o, self.batch, self.n_txt, self.n_img, self.heads, self.dim)
        ff.featfix_op_quant8("bf16", self.o, *self.a)
        self._linear("proj", self.a, out=self.d)
        ff.featfix_op_rms_norm("bf16", self.d, w["norm2"], self.eps, resid=x, sum_out=x, q=self.a[0], q_scale=self.a[1])
        self._linear("fc1", self.a, act=1, q=self.h[0], q_scale=self.h[1])
        self._linear("fc2", self.h, resid=x, out=x)
        return x
