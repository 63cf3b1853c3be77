"""Transformer layers in 8 bits that take one new token of each sequence at a time,
over an 8-bit cache of the keys and values of the earlier ones, built from the
operators of include/featfix_ops.h as a program uses them.  Per layer:

    qkv    = a Wqkv^T + b                                   featfix_op_gemm8
    q, k   = rotary positions on rms_norm(q), rms_norm(k)   featfix_op_rope
    cache  <- k, v in 8 bits                                featfix_op_kv_write
    o      = attention over the sequence's tokens           featfix_op_kv_attention
    d      = o (in 8 bits) Wproj^T + b                      featfix_op_quant8, featfix_op_gemm8
    x      = x + rms_norm(d);  a = rms_norm(x) in 8 bits    featfix_op_block_norms
    h      = GELU(a W1^T + b) in 8 bits                     featfix_op_gemm8
    d      = h W2^T + b                                     featfix_op_gemm8
    x      = x + rms_norm(d);  a = the next layer's rms_norm(x)   featfix_op_block_norms

with weights in all norms, and key heads that several query heads share.  Every
call of a step is asynchronous on the current stream and allocates nothing, and the
lengths and page tables are read on the device: a step that was captured in a graph
once serves all later ones.
"""

import operator

import torch

from . import featfix as ff
from .block8 import quantized

MATRICES = ("qkv", "proj", "fc1", "fc2")


class KVCache8:
    """Pages of 8-bit keys and values of ``layers`` layers, and who has which: the same
    page table and lengths serve every layer.  ``tokens``: the longest sequence.

    A step takes the last token of every sequence whose length is another than ``settled``, its length before it
    last grew; ``pending``: no step has run since.  All of them are on the GPU, where a captured step reads
    and leaves them."""

    def __init__(self, layers, pages, page_size, heads, dim, seqs, tokens, device="cuda"):
        pad = (dim + 15) // 16 * 16
        held = lambda: torch.zeros((layers, pages, page_size, heads, pad), dtype=torch.uint8, device=device)[..., :dim]
        scales = lambda: torch.zeros((layers, pages, page_size, heads), device=device)
        self.k8, self.v8, self.k_scale, self.v_scale = held(), held(), scales(), scales()
        self.page_size, self.width = page_size, -(-tokens // page_size)
        self.table = torch.full((seqs, self.width), -1, dtype=torch.int32, device=device)
        self.lens = torch.zeros(seqs, dtype=torch.int32, device=device)
        self.settled = torch.zeros(seqs, dtype=torch.int32, device=device)
        self.pending = torch.zeros((), dtype=torch.bool, device=device)
        self.free = list(range(pages - 1, -1, -1))
        self.held = [[] for _ in range(seqs)]
        self.used = [0] * seqs

    def layer(self, i):
        return self.k8[i], self.k_scale[i], self.v8[i], self.v_scale[i]

    def grow(self, counts):
        """Makes room for counts[b] more tokens of sequence b, as the next calls write them; asynchronous on the
        current stream, as the steps are.  Raises ValueError where counts are not one number from 0 on for each
        sequence, MemoryError where the pages or a sequence's row of the table run out, and changes nothing then."""
        try:
            counts = [operator.index(n) for n in counts]
        except TypeError:
            raise ValueError("counts: expected a whole number for each sequence")
        if len(counts) != len(self.used) or min(counts, default=0) < 0:
            raise ValueError("counts: expected %d numbers from 0 on" % len(self.used))
        used = [u + n for u, n in zip(self.used, counts)]
        need = [-(-u // self.page_size) for u in used]
        if max(need, default=0) > self.width or sum(n - len(h) for n, h in zip(need, self.held)) > len(self.free):
            raise MemoryError("no pages left for %d more tokens" % sum(counts))
        at, pages = [], []   # what changes in the table
        for b, n in enumerate(need):
            for i in range(len(self.held[b]), n):
                self.held[b].append(self.free.pop())
                at.append(b * self.width + i)
                pages.append(self.held[b][i])
        self.used = used
        # one copy from pinned memory: the host does not wait for the stream, as it would for pageable memory
        sent = torch.tensor(used + at + pages, dtype=torch.int64)
        if self.lens.is_cuda:
            sent = sent.pin_memory().to(self.lens.device, non_blocking=True)
        n, k = len(used), len(at)
        if k:
            self.table.view(-1)[sent[n:n + k]] = sent[n + k:].int()
        # (what grew twice since the last step is new from its first growth on)
        torch.where(self.pending, self.settled, self.lens, out=self.settled)
        self.pending.fill_(True)
        self.lens.copy_(sent[:n])

    def written(self):
        """A program wrote the tokens so far by itself: none of them is a step's new one."""
        self.settled.copy_(self.lens)

    def drop(self, b):
        """Sequence b is over: its pages are free again."""
        self.free += reversed(self.held[b])
        self.held[b], self.used[b] = [], 0
        self.lens[b].zero_()   # (an assignment would copy a number from the host, and wait)
        self.settled[b].zero_()
        self.table[b].fill_(-1)


class Step8:
    """Layers of one model.  ``layers``: a dict of bf16 GPU tensors for each: norm1 [C],
    qkv.w [(heads + 2 k_heads) d, C], qkv.b, q_norm [d], k_norm [d], proj.w [C, heads d], proj.b,
    norm1_after [C], norm2 [C], fc1.w [M, C], fc1.b, fc2.w [C, M], fc2.b, norm2_after [C]; the
    matrices are quantised here, once."""

    def __init__(self, layers, heads, k_heads, cache, theta=10000.0, eps=1e-6):
        self.w = [{k: v for k, v in w.items() if k.removesuffix(".w") not in MATRICES} for w in layers]
        self.q8 = [{m: quantized(w[m + ".w"]) for m in MATRICES} for w in layers]
        self.heads, self.k_heads, self.theta, self.eps, self.cache = heads, k_heads, theta, eps, cache
        n, (C, M) = cache.lens.numel(), layers[0]["fc2.w"].shape
        self.dim, dev = layers[0]["q_norm"].numel(), layers[0]["norm1"].device
        empty = lambda w: torch.empty((n, w), dtype=torch.bfloat16, device=dev)
        self.qkv, self.o, self.d = empty((heads + 2 * k_heads) * self.dim), empty(heads * self.dim), empty(C)
        self.pos = torch.empty((1, n), dtype=torch.int32, device=dev)
        # lengths of the sequences that have a new token, 0 of the others
        self.new, self.lens = torch.empty(n, dtype=torch.bool, device=dev), torch.empty(n, dtype=torch.int32, device=dev)
        # 8-bit activations with their scales: of width C, of the heads, of width M
        self.a, self.p, self.h = ((torch.zeros((n, (w + 15) // 16 * 16), dtype=torch.uint8, device=dev)[:, :w],
                                   torch.empty(((w + 127) // 128, n), dtype=torch.float32, device=dev))
                                  for w in (C, heads * self.dim, M))
        bytes_ = ff.featfix_op_kv_attention_workspace(n, heads, k_heads, self.dim, cache.width * cache.page_size)
        self.workspace = torch.empty(bytes_, dtype=torch.uint8, device=dev)

    def _linear(self, i, name, x, **kw):
        ff.featfix_op_gemm8("bf16", *x, *self.q8[i][name], bias=self.w[i][name + ".b"], **kw)

    def _norms(self, x, after, before):
        """x += norm(d) * after; the activations a = norm(x) * before, where there is a next norm."""
        to = {} if before is None else {"q": self.a[0], "q_scale": self.a[1]}
        ff.featfix_op_block_norms("bf16", self.d, x, self.eps, weight_after=after, sum_out=x, weight=before, **to)

    def __call__(self, x):
        """The residual stream x (bf16 [sequences, C]) of the last of each sequence's cache.lens
        tokens is updated in place.  A sequence that has no token, or none since the step before, is left out: its
        row means nothing, and nothing of it is written to the cache."""
        w, dim, c = self.w, self.dim, self.cache
        split = [n * dim for n in (self.heads, self.k_heads, self.k_heads)]
        q, k, v = self.qkv.split(split, 1)
        torch.ne(c.lens, c.settled, out=self.new)
        torch.mul(c.lens, self.new, out=self.lens)
        torch.sub(self.lens, 1, out=self.pos[0])
        ff.featfix_op_rms_norm("bf16", x, w[0]["norm1"], self.eps, q=self.a[0], q_scale=self.a[1])
        for i, wi in enumerate(w):
            self._linear(i, "qkv", self.a, out=self.qkv)
            ff.featfix_op_rope("bf16", self.pos, (dim,), dim, q=q, q_out=q, k=k, k_out=k, theta=self.theta,
                               q_weight=wi["q_norm"], k_weight=wi["k_norm"], eps=self.eps)
            ff.featfix_op_kv_write("bf16", k, v, c.layer(i), c.table, self.lens)
            ff.featfix_op_kv_attention("bf16", q, c.layer(i), c.table, self.lens, self.o, self.workspace, dim ** -0.5)
            ff.featfix_op_quant8("bf16", self.o, *self.p)
            self._linear(i, "proj", self.p, out=self.d)
            self._norms(x, wi["norm1_after"], wi["norm2"])
            self._linear(i, "fc1", self.a, act=1, q=self.h[0], q_scale=self.h[1])
            self._linear(i, "fc2", self.h, out=self.d)
            self._norms(x, wi["norm2_after"], w[i + 1]["norm1"] if i + 1 < len(w) else None)
        c.pending.fill_(False)
        return x
