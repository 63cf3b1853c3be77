"""Attention over the 8-bit cache where scores are large: every finite score of a row
has finite weights, whatever the sizes of the scores and of the values' scales are.

Keys of a row are one vector times a power of two to each token, so that products of equal
tokens are the same bits and other ones are far apart: the softmax is uniform over the
tokens of the largest score and zero elsewhere, exactly.  Then only values, their weights
and the sums round (bounds: kv_helpers.attention, with scores that are exact)."""

import pytest
import torch

from .kv_helpers import Cache, TD, U, quant
from .test_gpu_kv8 import attend, randn

pytestmark = pytest.mark.gpu


def rows(seqs, tokens, heads, group, dim, dtype, power, steps, spread, seed, sign=1.0):
    """A cache whose token t has the keys 2^(power + steps[t]) u; a query along u, others with at least half of a unit along it."""
    c = Cache(seqs * -(-tokens // 16) + 1, 16, heads, dim, seqs, -(-tokens // 16))
    c.place([tokens] * seqs, seed)
    c.fill(seed, spread)
    u, s = quant(randn((heads, dim), seed + 1))
    k = u.float() * s[:, None]
    q = randn((seqs, heads, group, dim), seed + 2)
    unit = (k / k.norm(dim=-1, keepdim=True))[None, :, None]
    along = randn((seqs, heads, group, 1), seed + 3)
    q += (along + torch.where(along < 0, -0.5, 0.5) - (q * unit).sum(-1, keepdim=True)) * unit
    q[:, :, 0] = k * sign
    for b in range(seqs):
        at = c.at(b, 0, tokens)
        c.k8[at] = u.view(torch.uint8).expand(tokens, heads, dim)
        c.k_scale[at] = torch.ldexp(s.expand(tokens, heads), (power + steps).int()[:, None])
    return c, q.view(seqs, -1).to(TD[dtype]), u.double() * s.double()[:, None]


def check(c, q, u, steps, scale, dtype):
    """Uniform over the tokens whose step is the largest where q u scale > 0, the smallest where it is below."""
    out, lse = attend(c, q, q.shape[1] // c.dim, scale)
    seqs, tokens, group = q.shape[0], steps.numel(), q.shape[1] // c.dim // c.heads
    along = torch.einsum("bhgd,hd->bhg", q.double().view(seqs, c.heads, group, c.dim), u) * scale
    assert (along.abs() > 0.25).all()
    for b in range(seqs):
        _, v = c.values(b, 0, tokens)
        for h in range(c.heads):
            for j in range(group):
                best = steps == (steps.max() if along[b, h, j] > 0 else steps.min())
                n, v1 = int(best.sum()), v[best][:, h]
                want, A = v1.mean(0), v1.abs().mean(0)
                rel = 2.0 ** -20 + (tokens + 64) * 2.0 ** -24 + (2.0 ** -11 if dtype == "bf16" else 2.0 ** -21)
                least = (2.0 ** -25 if dtype == "bf16" else 2.0 ** -36) * tokens * v1.abs().max() / n
                got = out[b].double().view(c.heads, group, c.dim)[h, j]
                assert ((got - want).abs() <= A * rel + least + want.abs() * U[dtype] * 1.01).all(), (b, h, j)
    assert lse.isfinite().all()
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("power", [20, 24, 25, 26, 27, 30, 41, 60, 100])
@pytest.mark.parametrize("seqs,tokens,heads,group,dim", [(8, 40, 4, 4, 128), (3, 500, 2, 8, 64), (1, 20000, 2, 4, 128), (2, 150, 1, 12, 96),
                                                         (2, 70, 2, 3, 256)])
def test_equal_scores_of_any_size(cuda, dtype, power, seqs, tokens, heads, group, dim):
    steps = torch.zeros(tokens, device="cuda")
    for sign in (1.0, -1.0):
        c, q, u = rows(seqs, tokens, heads, group, dim, dtype, power, steps, 1.0, power, sign)
        check(c, q, u, steps, dim ** -0.5, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("power", [20, 25, 26, 33, 60, 90])
@pytest.mark.parametrize("tokens", [33, 700, 20000])
def test_one_score_above_all(cuda, dtype, power, tokens):
    steps = torch.zeros(tokens, device="cuda")
    for at in (0, tokens // 3, tokens - 1):
        steps.zero_()
        steps[at] = 1
        c, q, u = rows(2, tokens, 2, 4, 128, dtype, power, steps, 2.0, power + at)
        check(c, q, u, steps, 128 ** -0.5, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("power,every", [(20, 40), (25, 7), (40, 300)])
@pytest.mark.parametrize("falling", [False, True])
def test_scores_that_rise_while_values_change(cuda, dtype, power, every, falling):
    """Every `every` tokens scores double and values halve, or double: the weights' common factor follows both."""
    tokens = 50 * every if every < 100 else 6000
    steps = (torch.arange(tokens, device="cuda") // every).clamp(max=40).float()
    c, q, u = rows(1, tokens, 2, 4, 64, dtype, power, steps, 0.5, every)
    at = c.at(0, 0, tokens)
    c.v_scale[at] = torch.ldexp(c.v_scale[at], (steps if falling else -steps).int()[:, None])
    check(c, q, u, steps, 0.125, dtype)


def test_queries_and_keys_of_1500(cuda):
    """Aligned queries and keys of this size have scores of 2^25 in heads of 128."""
    c, q, u = rows(32, 300, 2, 4, 128, "bf16", 0, torch.zeros(300, device="cuda"), 1.0, 3)
    c.k_scale.mul_(1500)
    out, lse = attend(c, q * 1500, 8)
    assert out.isfinite().all() and lse.isfinite().all()
    assert lse[0, 0] > 2.0 ** 24
    want = torch.stack([c.values(b, 0, 300)[1].mean(0) for b in range(32)])
    got = out.double().view(32, 2, 4, 128)
    A = torch.stack([c.values(b, 0, 300)[1].abs().mean(0) for b in range(32)])
    top = torch.stack([c.values(b, 0, 300)[1].abs().amax(0) for b in range(32)])
    tol = A * (2.0 ** -20 + 364 * 2.0 ** -24 + 2.0 ** -11) + 2.0 ** -25 * top + want.abs() * U["bf16"] * 1.01
    assert ((got - want[:, :, None]).abs() <= tol[:, :, None]).all()


@pytest.mark.parametrize("seqs,tokens,heads,group,dim", [(16, 40, 4, 4, 128), (8, 150, 2, 8, 64), (4, 150, 2, 12, 96), (1, 3000, 2, 4, 128),
                                                         (4, 70, 2, 3, 256)])
def test_bf16_results_are_those_of_fp32_weights(cuda, seqs, tokens, heads, group, dim):
    """Exact scores again, so that weights are the values' scales: a result is the rounding of a number within
    fp32's error, not bf16's, of the formula's."""
    steps = torch.zeros(tokens, device="cuda")
    c, q, u = rows(seqs, tokens, heads, group, dim, "bf16", 3, steps, 1.0, 7)
    out, _ = attend(c, q, heads * group, dim ** -0.5)
    got = out.view(seqs, heads, group, dim)
    for b in range(seqs):
        _, v = c.values(b, 0, tokens)
        want, A, top = v.mean(0)[:, None], v.abs().mean(0)[:, None], v.abs().amax(0)[:, None]
        e = A * (2.0 ** -20 + (tokens + 64) * 2.0 ** -24 + 2.0 ** -21) + 2.0 ** -36 * top
        assert ((got[b] >= (want - e).bfloat16()) & (got[b] <= (want + e).bfloat16())).all()
