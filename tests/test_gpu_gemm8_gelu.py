"""The GELU of the 8-bit product over all arguments, in both kernels, against float64.

A has only zeros, so a column's argument is its bias, exactly.  Bounds: the result is
within |x| 2^-20 of the exact one near zero and for positive x (a few fp32 roundings of
the argument), and within 1e-6 for negative x, where the exact value goes back to zero."""

import math

import pytest
import torch

from paper_2607_27842_gb300 import featfix as ff

from .test_gpu_ops8 import F8, TD, U, gelu64, held, held8, nb, values

pytestmark = pytest.mark.gpu


def product_of_zeros(dtype, M, N, K, bias, q8=False):
    a, w = (torch.zeros((n, (K + 15) // 16 * 16), dtype=torch.uint8, device="cuda").view(F8)[:, :K] for n in (M, N))
    sa, sw = torch.ones((nb(K), M), device="cuda"), torch.ones((nb(N), nb(K)), device="cuda")
    if q8:
        q, s = held8(M, N), torch.empty((nb(N), M), device="cuda")
        ff.featfix_op_gemm8(dtype, a, sa, w, sw, bias=bias, act=1, q=q, q_scale=s)
        return values(q, s, 1)
    out = held(M, N, TD[dtype])
    ff.featfix_op_gemm8(dtype, a, sa, w, sw, out=out, bias=bias, act=1)
    return out


# few rows (the product transposed) and CTA pairs
SIZES = [(3, 500, 16), (6000, 2050, 200)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_gelu_of_every_magnitude(cuda, dtype, M, N, K):
    """-2^127 to -2^-6 and the same positive, in an order that mixes them in every four."""
    x = 2.0 ** torch.linspace(-6, 127, N // 2, dtype=torch.float64)
    x = torch.cat([-x, x])[torch.randperm(N, generator=torch.Generator().manual_seed(1))].to(TD[dtype]).cuda()
    y = x.double()
    want = torch.where(y < -40, torch.zeros_like(y), torch.where(y > 40, y, gelu64(y.clamp(-40, 40))))
    out = product_of_zeros(dtype, M, N, K, x)
    tol = want.abs() * U[dtype] * 1.01 + torch.where(y < 0, torch.full_like(y, 1e-6), y * 2.0 ** -20)
    assert ((out.double() - want).abs() <= tol).all(), float(((out.double() - want).abs() / tol).max())


@pytest.mark.parametrize("M,N,K", SIZES)
def test_gelu_of_large_negative_rows_in_8_bits(cuda, M, N, K):
    """All of a block far below zero: its values vanish with its scale."""
    x = -(10.0 ** torch.linspace(1.5, 30, N, dtype=torch.float64)).float().cuda()
    assert (product_of_zeros("f32", M, N, K, x, q8=True).abs() <= 1e-6).all()


@pytest.mark.parametrize("M,N,K", SIZES)
def test_gelu_of_infinities_and_nan(cuda, M, N, K):
    """As the formula has it: infinity stays, minus infinity times zero and NaN are NaN;
    the columns beside them keep their values."""
    g = torch.Generator().manual_seed(2)
    x = torch.randn(N, generator=g).cuda()
    plain = product_of_zeros("f32", M, N, K, x).clone()
    y = x.clone()
    y[5::16], y[6::16], y[8::32] = math.inf, -math.inf, math.nan
    out = product_of_zeros("f32", M, N, K, y)
    assert (out[:, 5::16] == math.inf).all()
    assert torch.isnan(out[:, 6::16]).all() and torch.isnan(out[:, 8::32]).all()
    keep = torch.isfinite(y)
    # (a row's values are formed four at a time; a special one among them costs the rest nothing)
    assert ((out[:, keep] - plain[:, keep]).abs() <= x[keep].abs() * 2.0 ** -20).all()
