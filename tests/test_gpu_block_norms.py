"""The norms before and after a block with gate and residual (featfix_op_block_norms)
through the C ABI against the formula in float64.

Bounds, per row of C columns.  norm(u) = (u - mean) r: r is off by at most (C + 8) 2^-25 +
2^-21 relative to itself (half of its sum's error, and rsqrt), the mean by (C + 8) 2^-24 of the
largest |u|, in the worst case of adding one after the other; errors e of u itself come through as
(e + the mean's + |norm(u)| times their root mean square) r.  Every product and sum adds 2^-24 of
its result."""

import pytest
import torch

from paper_2607_27842_gb300 import featfix as ff

from .test_gpu_ops8 import TD, check, check8, held, held8, nb, randn, untouched

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


def norm(u, e, w, eps, centered):
    """norm(u) * w and its bound, for u off by at most e."""
    C = u.shape[1]
    rms = lambda t: (t * t).mean(-1, keepdim=True).sqrt()
    d = u - u.mean(-1, keepdim=True) if centered else u
    em = e.mean(-1, keepdim=True) + (C + 8) * E * u.abs().amax(-1, keepdim=True) if centered else 0
    r = 1 / torch.sqrt((d * d).mean(-1, keepdim=True) + eps)
    y = d * r
    ed = e + em + d.abs() * E
    err = (ed + y.abs() * rms(ed + 0 * d)) * r + y.abs() * ((C + 8) * E / 2 + 2.0 ** -21)
    w = torch.ones_like(u[0]) if w is None else w.double()
    return y * w, (err + 2 * y.abs() * E) * w.abs()


def formula(t, eps, resid_scale, after, centered, rpb, rows):
    """(h, its bound, z, its bound)."""
    d = lambda n: t[n].double()
    of = torch.arange(rows, device="cuda") // max(rpb, 1)
    h, e = d("y"), torch.zeros_like(d("y"))
    if after:
        h, e = norm(h, e, t.get("weight_after"), eps, centered)
    if "gate" in t:
        g = d("gate")[of]
        h, e = h * g, e * g.abs() + (h * g).abs() * E
    if "x" in t:
        x = resid_scale * d("x")
        h, e = h + x, e + (x.abs() + (h + x).abs()) * E
    z, ez = norm(h, e, t.get("weight"), eps, centered)
    if "scale" in t:
        s = 1 + d("scale")[of]
        z, ez = z * s, ez * s.abs() + 2 * (z * s).abs() * E
    if "shift" in t:
        z = z + d("shift")[of]
        ez = ez + z.abs() * E + d("shift")[of].abs() * E
    return h, e, z, ez


def inputs(rows, C, td, extra, samples, seed, which):
    t = {}
    for i, n in enumerate(("y", "x")):
        if n in which:
            t[n] = held(rows, C, td, extra)
            t[n].copy_(randn((rows, C), seed + i, 2.0) + (3.0 if n == "y" else 0.5))
    for i, n in enumerate(("weight_after", "weight")):
        if n in which:
            t[n] = (1 + randn((C,), seed + 5 + i, 0.3)).to(td)
    mod = randn((samples, 6 * C), seed + 9, 0.5)
    for i, n in enumerate(("gate", "shift", "scale")):
        if n in which:
            t[n] = mod[:, (i + 2) * C:(i + 3) * C]
    return t


ALL = ("y", "x", "weight_after", "weight", "gate", "shift", "scale")


def run(dtype, t, eps=1e-6, resid_scale=0.9, after=True, centered=False, rpb=0, result="out", extra=0, sum_out=True):
    rows, C = t["y"].shape
    td, got = TD[dtype], {}
    if sum_out:
        got["sum_out"] = held(rows, C, td, extra)
    if result == "out":
        got["out"] = held(rows, C, td, extra)
    if result == "q":
        got["q"], got["q_scale"] = held8(rows, C, 16), torch.full((nb(C), rows), 3.0, device="cuda")
    ff.featfix_op_block_norms(dtype, t["y"], t.get("x"), eps, weight_after=t.get("weight_after"), norm_after=after,
                              resid_scale=resid_scale, gate=t.get("gate"), weight=t.get("weight"), shift=t.get("shift"),
                              scale=t.get("scale"), rows_per_batch=rpb, centered=centered, **got)
    torch.cuda.synchronize()
    h, e, z, ez = formula(t, eps, resid_scale, after, centered, rpb, rows)
    if sum_out:
        check(got["sum_out"], h, dtype, e)
        assert untouched(got["sum_out"])
    if result == "out":
        check(got["out"], z, dtype, ez)
        assert untouched(got["out"])
    if result == "q":
        check8(got["q"], got["q_scale"], z, 1, ez)
        assert untouched(got["q"])
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("result", ["out", "q"])
@pytest.mark.parametrize("centered", [False, True])
@pytest.mark.parametrize("rows,C,extra,rpb", [
    (1, 1, 0, 1), (3, 8, 8, 2), (5, 127, 1, 5), (2, 129, 0, 1), (1, 2048, 0, 7), (333, 1000, 24, 100), (700, 1152, 0, 333),
    (9, 1160, 8, 4), (40, 5120, 0, 13), (3, 8200, 0, 2), (2, 16384, 0, 1), (4, 16001, 0, 4), (1500, 64, 0, 7), (5000, 256, 0, 4999),
    (4099, 2048, 0, 2050), (6001, 72, 0, 1), (2600, 1001, 1, 600), (3000, 4096, 0, 2999)])
def test_block_norms(cuda, dtype, result, centered, rows, C, extra, rpb):
    t = inputs(rows, C, TD[dtype], extra, -(-rows // rpb), 31, ALL)
    run(dtype, t, centered=centered, rpb=rpb, result=result, extra=extra)


WITHOUT = [("x",), ("gate",), ("weight_after", "weight"), ("shift",), ("scale",), ("gate", "shift", "scale"), ("x", "gate"),
           ("weight_after",), ("weight", "shift", "scale"), ("x", "gate", "weight", "shift", "scale", "weight_after")]


@pytest.mark.parametrize("rows,C", [(37, 1152), (2000, 200), (70, 333)])
@pytest.mark.parametrize("without", WITHOUT)
@pytest.mark.parametrize("after", [False, True])
def test_parts_that_are_absent(cuda, without, after, rows, C):
    drop = set(without) | (set() if after else {"weight_after"})
    t = inputs(rows, C, torch.bfloat16, 0, -(-rows // 30), 41, [n for n in ALL if n not in drop])
    rpb = 30 if drop.isdisjoint({"gate", "shift", "scale"}) or {"gate", "shift", "scale"} - drop else 0
    for i, result in enumerate(("out", "q", None)):
        run("bf16", t, after=after, centered=i == 1, rpb=rpb, result=result, sum_out=i != 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C", [(3000, 1152), (5, 9000), (64, 77)])
def test_in_place(cuda, dtype, rows, C):
    """The sum over x, the result over y; then the sum over y."""
    t = inputs(rows, C, TD[dtype], 0, 2, 51, ALL)
    rpb = -(-rows // 2)
    args = dict(weight_after=t["weight_after"], gate=t["gate"], weight=t["weight"], shift=t["shift"], scale=t["scale"],
                rows_per_batch=rpb)
    s, o = torch.empty_like(t["x"]), torch.empty_like(t["x"])
    ff.featfix_op_block_norms(dtype, t["y"], t["x"], 1e-6, sum_out=s, out=o, **args)
    x, y = t["x"].clone(), t["y"].clone()
    ff.featfix_op_block_norms(dtype, y, x, 1e-6, sum_out=x, out=y, **args)
    assert (x == s).all() and (y == o).all()
    y = t["y"].clone()
    ff.featfix_op_block_norms(dtype, y, t["x"], 1e-6, sum_out=y, **args)
    assert (y == s).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_unaligned_rows_and_broadcast_modulation(cuda, dtype):
    """Rows, weights and modulation rows off a vector's boundary give what aligned ones give, up to
    the order of a sum."""
    rows, C = 500, 768
    base = held(rows, 4 * C + 5, TD[dtype])
    base.copy_(randn(base.shape, 61))
    mod = randn((3, 3 * C + 3), 62, 0.4)
    w = (1 + randn((2 * C + 2,), 63, 0.2)).to(TD[dtype])
    t = {"y": base[:, 1:C + 1], "x": base[:, C + 2:2 * C + 2], "weight_after": w[1:C + 1], "weight": w[C + 2:],
         "gate": mod[:, 1:C + 1], "shift": mod[:, C + 1:2 * C + 1], "scale": mod[:, 2 * C + 3:3 * C + 3]}
    for result in ("out", "q"):
        run(dtype, t, rpb=200, result=result)
        run(dtype, t, rpb=200, result=result, centered=True)


def test_large_means_and_special_rows(cuda):
    """A mean 10^4 times the deviation keeps its digits; a NaN, an infinity or zeros stay in their
    row."""
    rows, C = 64, 1536
    t = inputs(rows, C, torch.float32, 0, 1, 71, ("y", "x", "weight"))
    t["x"] += 2e4
    run("f32", t, centered=True, after=False)
    t = inputs(rows, C, torch.float32, 0, 1, 72, ("y", "x"))
    t["y"][3, 5], t["x"][7, 1000], t["y"][9], t["x"][9] = float("nan"), float("inf"), 0, 0
    out, s = torch.empty_like(t["y"]), torch.empty_like(t["y"])
    q, qs = held8(rows, C), torch.empty((nb(C), rows), device="cuda")
    ff.featfix_op_block_norms("f32", t["y"], t["x"], 1e-6, sum_out=s, out=out)
    ff.featfix_op_block_norms("f32", t["y"], t["x"], 1e-6, q=q, q_scale=qs)
    assert out[3].isnan().all() and out[7].isnan().any() and (out[9] == 0).all() and (s[9] == 0).all()
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
    bad[[3, 7]] = True
    assert out[~bad].isfinite().all() and qs[:, ~bad].isfinite().all() and qs[:, 3].isnan().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C,extra", [(4099, 2048, 0), (2501, 1001, 1), (700, 8192, 0), (300, 16384, 0), (305, 9001, 0)])
@pytest.mark.parametrize("after", [False, True])
def test_one_norm_to_a_row(cuda, dtype, rows, C, extra, after):
    """Rows of several warps with a single norm each (the one before the block, or the one after it and the sum
    alone): sums of adjacent rows, a thousandfold apart, do not meet."""
    t = inputs(rows, C, TD[dtype], extra, 1, 51, ("y", "x") if after else ("y", "weight"))
    t["y"][::2] *= 1000
    first = run(dtype, t, after=after, result=None if after else "out", extra=extra, sum_out=after)
    for _ in range(5):
        again = run(dtype, t, after=after, result=None if after else "out", extra=extra, sum_out=after)
        assert all((again[n] == first[n]).all() for n in first)


def test_no_rows(cuda):
    x = torch.empty((0, 64), device="cuda")
    n0 = ff.featfix_launch_count()
    ff.featfix_op_block_norms("f32", x, x, 1e-6, out=x)
    assert ff.featfix_launch_count() == n0
