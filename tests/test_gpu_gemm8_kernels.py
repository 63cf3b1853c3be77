"""Every kernel of the 8-bit product that a call can reach, and the places where its
loops turn over, against float64 (bounds: test_gpu_ops8.py)."""

import pytest
import torch

from paper_2607_27842_gb300 import featfix as ff

from .test_gpu_ops8 import TD, check, check8, gelu64, gemm_inputs, gemm_ref, held, held8, nb, randn, untouched


def plan(M, N, K, sms):
    """(rows of A to a tile, CTAs to a cluster) of the split kernel or (0, 1), CTA pairs:
    the dispatch's time model restated, and the least time of the kernels not taken."""
    ceil = lambda a, b: -(-a // b)
    kb = ceil(K, 128)
    times = {(0, 1): ceil(ceil(M, 256) * ceil(N, 256), sms // 2) * (0.549 * kb + 3.65) + 4.7}
    for i, bt in enumerate((16, 32, 64)):
        if i and bt // 2 >= M:
            break
        for l in range(4):
            if 1 << l > kb:
                break
            ctas = ceil(N, 128) * ceil(M, bt) << l
            shared = ctas > sms
            each = ((0.300, 0.467, 0.558) if shared else (0.321, 0.381, 0.365))[i] * ceil(kb, 1 << l) + (1.73, 2.15, 5.57)[i]
            times[bt, 1 << l] = (ceil(ctas, 2 * sms) * each + 2.0 + (0, 0.27, 0.23, 0.44)[l] + (0.61 if shared else 0) +
                                 0.18 * min(1.0, ctas / (2 * sms)))
    best = min(times, key=times.get)
    return best, min((t for p, t in times.items() if p != best), default=float("inf")) / times[best]


# M, N, K and the kernel at 148 and at 152 SMs
SIZES = [
    (256, 2048, 8192, (64, 4), (64, 4)),      # partial sums in the peers' rings
    (250, 2050, 8190, (64, 4), (64, 4)),      # the same, ragged
    (512, 2048, 8192, (64, 2), (64, 2)),      # one whole table of scales (32 blocks of K to a CTA)
    (56, 10178, 10492, (64, 2), (64, 2)),     # a second table begins (41 blocks)
    (572, 2086, 507, (64, 1), (64, 1)),
    (1319, 29, 15957, (64, 8), (64, 8)),
    (300, 2048, 8192, (64, 2), (16, 1)),      # 64 blocks of K to a CTA of 16 rows at 152 SMs
    (41, 10304, 4215, (16, 1), (16, 1)),      # 33 blocks: a second table of one
    (3, 9763, 2204, (16, 2), (16, 2)),
    (14, 665, 646, (16, 4), (16, 4)),
    (1, 75, 15886, (16, 8), (16, 8)),
    (1400, 10, 19, (16, 1), (16, 1)),
    (1077, 1000, 712, (32, 1), (32, 1)),
    (18, 14764, 8277, (32, 2), (32, 2)),      # 33 blocks
    (2032, 33, 5277, (32, 4), (32, 4)),
    (839, 107, 10849, (32, 8), (32, 8)),
    (1500, 2300, 2100, (0, 1), (0, 1)),       # pairs: the ring of four blocks of K turns over
    (2600, 2050, 2333, (0, 1), (0, 1)),       # and over several tiles
    (996, 9108, 1034, (0, 1), (0, 1)),
]


@pytest.mark.parametrize("sms", [148, 152])
def test_sizes_reach_their_kernels(sms):
    for M, N, K, at148, at152 in SIZES:
        assert plan(M, N, K, sms)[0] == (at148 if sms == 148 else at152), (M, N, K, plan(M, N, K, sms))
    reached = {plan(*c[:3], sms)[0] for c in SIZES}
    assert reached == {(0, 1)} | {(bt, s) for bt in (16, 32, 64) for s in (1, 2, 4, 8)}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [c[:3] for c in SIZES])
def test_gemm8_kernels(cuda, dtype, M, N, K):
    td = TD[dtype]
    a, sa, w, sw = gemm_inputs(M, N, K, 20, 16, 32)
    ref, mag = gemm_ref(a, sa, w, sw)
    err = mag * (128 + nb(K) + 4) * 2.0 ** -24
    out = held(M, N, td, 8)
    ff.featfix_op_gemm8(dtype, a, sa, w, sw, out=out)
    check(out, ref, dtype, err)
    assert untouched(out)
    bias = randn((N,), 23).to(td)
    y = ref + bias.double()
    gate, rpb = randn((-(-M // 100), 2 * N), 24)[:, N:], 100
    resid = held(M, N, td, 8)
    resid.copy_(randn((M, N), 25, 2.0))
    gm = gate.double().repeat_interleave(rpb, 0)[:M]
    want = resid.double() + gm * y
    terr = gm.abs() * (err + y.abs() * 2.0 ** -23) + want.abs() * 2.0 ** -23
    ff.featfix_op_gemm8(dtype, a, sa, w, sw, out=resid, bias=bias, gate=gate, rows_per_batch=rpb, resid=resid)
    check(resid, want, dtype, terr)
    assert untouched(resid)
    first = resid.clone()
    g = gelu64(y)
    q, s = held8(M, N, 16), torch.empty((nb(N), M), device=cuda)
    ff.featfix_op_gemm8(dtype, a, sa, w, sw, bias=bias, act=1, q=q, q_scale=s)
    check8(q, s, g, 1, 1.13 * err + y.abs() * 2.0 ** -20)
    assert untouched(q)
    resid.copy_(randn((M, N), 25, 2.0))
    ff.featfix_op_gemm8(dtype, a, sa, w, sw, out=resid, bias=bias, gate=gate, rows_per_batch=rpb, resid=resid)
    assert torch.equal(resid, first)                           # the same bits again
    ff.featfix_op_gemm8_watchdog()
