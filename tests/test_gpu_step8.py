"""Layers that take one new token of each sequence (step8.Step8) against the same
layers in float64 over all tokens at once, without any rounding.

Bound.  As for the block without a cache: e4m3 leaves 2^-4 / sqrt(3) of a product's operands in the
root mean square, so each of a layer's four products 2^-4 sqrt(2 / 3) = 0.051 of its result; keys,
values and the attention's output are rounded once each, at most 0.036 each of what the attention
gives, together 0.062; and bf16 steps.  Norms after a block keep the ratio.  What one layer adds is
held to 5 * 0.051 + 0.062, of two layers to twice that."""

import math

import pytest
import torch

from paper_2607_27842_gb300 import step8

pytestmark = pytest.mark.gpu


def weights(C, M, heads, k_heads, dim, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *d, s=1.0: (torch.randn(d, generator=g) * s).bfloat16().cuda()
    one = lambda n: (1 + 0.2 * torch.randn(n, generator=g)).bfloat16().cuda()
    s, n = 1 / math.sqrt(C), (heads + 2 * k_heads) * dim
    return {"norm1": one(C), "qkv.w": r(n, C, s=s), "qkv.b": r(n, s=0.1), "q_norm": one(dim), "k_norm": one(dim),
            "proj.w": r(C, heads * dim, s=1 / math.sqrt(heads * dim)), "proj.b": r(C, s=0.1), "norm1_after": one(C),
            "norm2": one(C), "fc1.w": r(M, C, s=s), "fc1.b": r(M, s=0.1), "fc2.w": r(C, M, s=1 / math.sqrt(M)),
            "fc2.b": r(C, s=0.1), "norm2_after": one(C)}


def plain(x, layers, heads, k_heads, eps=1e-6, theta=10000.0):
    """All tokens [n, C] of one sequence at once, each seeing itself and those before it."""
    x, n = x.double(), x.shape[0]
    norm = lambda v, g: v / torch.sqrt((v * v).mean(-1, keepdim=True) + eps) * g
    for w in layers:
        w = {k: v.double() for k, v in w.items()}
        dim = w["q_norm"].numel()
        linear = lambda v, m: v @ w[m + ".w"].t() + w[m + ".b"]
        ang = (torch.arange(n, device=x.device).double()[:, None] *
               theta ** (-2 * torch.arange(dim // 2, device=x.device).double() / dim))[:, None]

        def turned(v, g):
            v = norm(v, g)
            a, b = v[..., 0::2], v[..., 1::2]
            return torch.stack([a * ang.cos() - b * ang.sin(), a * ang.sin() + b * ang.cos()], -1).flatten(-2)

        q, k, v = linear(norm(x, w["norm1"]), "qkv").view(n, -1, dim).split([heads, k_heads, k_heads], 1)
        q, k, v = turned(q, w["q_norm"]), turned(k, w["k_norm"]).repeat_interleave(heads // k_heads, 1), \
            v.repeat_interleave(heads // k_heads, 1)
        s = torch.einsum("nhd,mhd->hnm", q, k) / math.sqrt(dim)
        s = s.masked_fill(torch.ones(n, n, device=x.device).triu(1).bool(), -math.inf)
        o = torch.einsum("hnm,mhd->nhd", torch.softmax(s, -1), v).reshape(n, -1)
        x = x + norm(linear(o, "proj"), w["norm1_after"])
        h = linear(norm(x, w["norm2"]), "fc1")
        h = 0.5 * h * (1 + torch.tanh(math.sqrt(2 / math.pi) * (h + 0.044715 * h ** 3)))
        x = x + norm(linear(h, "fc2"), w["norm2_after"])
    return x


@pytest.mark.parametrize("heads,k_heads,dim,page,n_layers", [(4, 4, 64, 16, 1), (8, 2, 64, 4, 2), (6, 1, 72, 7, 1),
                                                            (16, 4, 128, 64, 1)])
def test_steps(cuda, heads, k_heads, dim, page, n_layers):
    C, M, steps, seqs = heads * dim, 2 * heads * dim, 24, 3
    layers = [weights(C, M, heads, k_heads, dim, 80 + i) for i in range(n_layers)]
    cache = step8.KVCache8(n_layers, 3 * seqs * (-(-steps // page)), page, k_heads, dim, seqs, steps)
    model = step8.Step8(layers, heads, k_heads, cache)
    x = torch.randn((steps, seqs, C), generator=torch.Generator().manual_seed(90)).bfloat16().cuda()
    # sequence 1 begins 5 steps later; sequence 2 ends after 10 and another one takes its place
    first = [0, 5, 10]
    got = {}
    buf, graph = x[0].clone(), None
    for i in range(steps):
        cache.grow([1, int(i >= 5), 1])
        buf.copy_(x[i])
        if i == 10:
            cache.drop(2)
            cache.grow([0, 0, 1])
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                model(buf)
            buf.copy_(x[i])
        if graph:
            graph.replay()
        else:
            model(buf)
        got[i] = buf.double()
    for b in range(seqs):
        xs = x[first[b]:, b]
        want = plain(xs, layers, heads, k_heads)
        mine = torch.stack([got[i][b] for i in range(first[b], steps)])
        added, err = (want - xs.double()).norm(), (mine - want).norm()
        assert err <= n_layers * (5 * 0.051 + 0.062) * added, (b, float(err / added))


def test_pages(cuda):
    cache = step8.KVCache8(1, 5, 4, 1, 64, 2, 16)
    cache.grow([4, 9])
    assert sorted(cache.held[0] + cache.held[1]) == sorted(set(cache.held[0] + cache.held[1])) and len(cache.free) == 1
    before = (list(cache.used), cache.table.clone())
    for bad in ([1, 4], [13, 0]):
        with pytest.raises(MemoryError):
            cache.grow(bad)
    assert cache.used == before[0] and (cache.table == before[1]).all()
    cache.drop(1)
    assert len(cache.free) == 4 and cache.lens.tolist() == [4, 0]
    cache.grow([12, 0])
    assert cache.lens.tolist() == [16, 0] and len(set(cache.held[0])) == 4
