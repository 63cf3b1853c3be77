"""Caches, their plain reading and plain attention in float64, for the tests of the
8-bit key-value cache."""

import math

import torch

F8 = torch.float8_e4m3fn
TD = {"f32": torch.float32, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
NAN8 = 0x7f            # e4m3's NaN: what places and padding hold that nothing may read


class Cache:
    """A cache whose every byte is NaN until it is written.  ``layout`` "token": [pages, slots,
    heads]; "head": [pages, heads, slots]; "gap": as token with room between the places.
    Table places behind a sequence's end hold numbers of no page."""

    def __init__(self, pages, page, heads, dim, seqs, table_pages, layout="token", device="cuda"):
        self.pages, self.page, self.heads, self.dim = pages, page, heads, dim
        self.k8, self.k_scale = self.pool(layout, device)
        self.v8, self.v_scale = self.pool(layout, device)
        self.table = torch.full((seqs, table_pages), 1 << 30, dtype=torch.int32, device=device)
        self.lens = torch.zeros(seqs, dtype=torch.int32, device=device)

    def pool(self, layout, device):
        pad, gap = (self.dim + 15) // 16 * 16, 32 if layout == "gap" else 0
        size = (self.pages, self.heads, self.page) if layout == "head" else (self.pages, self.page, self.heads)
        q = torch.full(size + (pad + gap,), NAN8, dtype=torch.uint8, device=device)[..., :self.dim]
        s = torch.full(size + (1 + gap // 16,), math.nan, device=device)[..., 0]
        return (q.transpose(1, 2), s.transpose(1, 2)) if layout == "head" else (q, s)

    @property
    def parts(self):
        return self.k8, self.k_scale, self.v8, self.v_scale

    def place(self, lens, seed=0):
        """Pages in random order for sequences of these lengths."""
        g = torch.Generator().manual_seed(seed)
        need = [-(-n // self.page) for n in lens]
        order = torch.randperm(self.pages, generator=g)[:sum(need)].to(torch.int32)
        assert len(order) == sum(need)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n].to(self.table.device)
            at += n
        self.lens.copy_(torch.tensor(lens, dtype=torch.int32))

    def at(self, b, first, end):
        t = torch.arange(first, end, device=self.table.device)
        return self.table[b, t // self.page].long(), t % self.page

    def fill(self, seed=1, spread=0.5):
        """Values and scales for all tokens of all sequences, the scales of tokens e^spread apart."""
        g = torch.Generator().manual_seed(seed)
        for b, n in enumerate(self.lens.tolist()):
            if n == 0:
                continue
            at = self.at(b, 0, n)
            for q, s in ((self.k8, self.k_scale), (self.v8, self.v_scale)):
                x = torch.randn((n, self.heads, self.dim), generator=g)
                scale = torch.exp(torch.randn((n, self.heads), generator=g) * spread) / 100
                q[at] = (x * 100).clamp(-448, 448).to(F8).view(torch.uint8).to(q.device)
                s[at] = scale.to(s.device)

    def values(self, b, first, end):
        """k, v [tokens, heads, dim] in float64; a missing page's tokens are NaN."""
        page, slot = self.at(b, first, end)
        there = (page >= 0) & (page < self.pages)
        page = torch.where(there, page, 0)
        out = []
        for q, s in ((self.k8, self.k_scale), (self.v8, self.v_scale)):
            x = q[page, slot].view(F8).double() * s[page, slot].double()[..., None]
            out.append(torch.where(there[:, None, None], x, math.nan))
        return out


def quant(x):
    """Values and fp32 scale of each vector of the last dimension, in float64 arithmetic."""
    s = (x.double().abs().amax(-1) / 448).clamp(min=2.0 ** -100).float()
    return (x.double() / s[..., None].double()).clamp(-448, 448).float().to(F8), s


def attention(cache, q, q_heads, scale, window, dtype):
    """(out, lse, bound of out's error, bound of lse's) in float64.

    With X = scale sum |q_i k_i|, a score is off by at most X (dim + 8) 2^-24 from fp32 sums,
    by X 2^-21 from q in two fp16 terms (bf16: by 2^-25 of its largest magnitude for each of
    its elements) and by |x| 2^-22 from its rounding; a probability by twice the largest of
    these relative to itself, 2^-20 for the exponential, and its own rounding (2^-11 in one fp16
    term, 2^-21 in two); weights a factor of 2^14 below the largest lose 2^-25 of that one at
    most.  Sums of n tokens in fp32: n 2^-24 of the sum of magnitudes."""
    dim, group = cache.dim, q_heads // cache.heads
    rows = []
    for b, n in enumerate(cache.lens.tolist()):
        n = max(0, min(n, cache.table.shape[1] * cache.page))
        first = max(0, n - window) if window else 0
        qb = q[b].double().view(q_heads, dim)
        out, lse = torch.zeros((q_heads, dim)).double().to(q.device), torch.full((q_heads,), -math.inf).double().to(q.device)
        eo, el = torch.zeros_like(out), torch.zeros_like(lse)
        if n > first:
            k, v = cache.values(b, first, n)
            there = ~k.isnan().all(-1).all(-1)
            k, v, m = k[there], v[there], int(there.sum())
        if n > first and m:
            k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
            x = torch.einsum("hd,thd->ht", qb, k) * scale
            X = torch.einsum("hd,thd->ht", qb.abs(), k.abs()) * abs(scale)
            low = 2.0 ** -21 * X if dtype == "f32" else 2.0 ** -25 * qb.abs().amax(1)[:, None] * k.abs().sum(-1).t() * abs(scale)
            dx = ((dim + 8) * 2.0 ** -24 * X + low + x.abs() * 2.0 ** -22).amax(1)
            p = torch.softmax(x, 1)
            out, lse = torch.einsum("ht,thd->hd", p, v), torch.logsumexp(x, 1)
            A = torch.einsum("ht,thd->hd", p, v.abs())
            rel = 2 * dx + 2.0 ** -20 + (m + 64) * 2.0 ** -24 + (2.0 ** -11 if dtype == "bf16" else 2.0 ** -21)
            least = 2.0 ** -25 if dtype == "bf16" else 2.0 ** -36
            W = (p * v.abs().amax(-1).t()).amax(1)
            eo = A * rel[:, None] + m * least * W[:, None] + out.abs() * U[dtype] * 1.01
            el = dx + (m + 64) * 2.0 ** -24 + lse.abs() * 2.0 ** -22 + 2.0 ** -20
        rows.append((out.flatten(), lse, eo.flatten(), el))
    return tuple(torch.stack(r) for r in zip(*rows))
