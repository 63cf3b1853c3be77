"""The operators of the 8-bit layers (norm, quantiser, product, rotary
positions) through the C ABI, each against its formula in float64.

Bounds.  u16 = 2^-8 and u8 = 2^-4 are the unit roundoffs of bf16 and e4m3 (8 and 4
significant bits), and 2^-10 half the step of e4m3's denormals.  fp32 sums of n
terms are held to the worst case n 2^-24 of the sum of magnitudes, elementwise
results to a few 2^-24 of theirs.
"""

import math

import pytest
import torch

from paper_2607_27842_gb300 import featfix as ff

pytestmark = pytest.mark.gpu

TD = {"f32": torch.float32, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
F8 = torch.float8_e4m3fn


def randn(dims, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(dims, generator=g) * scale).cuda()


def pad16(n):
    return (n + 15) // 16 * 16


def nb(n):
    return (n + 127) // 128


def held(rows, cols, td, extra=0):
    """A [rows, cols] view of rows `extra` elements longer, filled with a
    pattern that a stray write disturbs."""
    return torch.full((rows, cols + extra), 3.0, device="cuda").to(td)[:, :cols]


def held8(rows, cols, extra=0):
    return torch.full((rows, pad16(cols) + extra), 0x55, dtype=torch.uint8, device="cuda").view(F8)[:, :cols]


def untouched(view):
    """The columns past a view's width still hold what held / held8 put there."""
    base = view._base if view._base.dim() == 2 else view
    rest = torch.as_strided(view, (view.shape[0], max(0, view.stride(0) - view.shape[1])), (view.stride(0), 1),
                            view.storage_offset() + view.shape[1])
    if rest.numel() == 0:
        return True
    if view.dtype == F8:
        return bool((rest.contiguous().view(torch.uint8) == 0x55).all())
    return bool((rest.float() == 3.0).all())


def quant(x, tile):
    """Reference quantisation in float64, scales in the ABI's layout and fp32."""
    rows, cols = x.shape
    p = torch.nn.functional.pad(x.double(), (0, -cols % 128, 0, -rows % tile))
    v = p.view(p.shape[0] // tile, tile, -1, 128)
    s = (v.abs().amax(dim=(1, 3)) / 448).clamp(min=2.0 ** -100).float()
    q = (v / s[:, None, :, None].double()).clamp(-448, 448).float().to(F8).view(p.shape)[:rows, :cols]
    buf = held8(rows, cols)
    buf.copy_(q)
    return buf, s if tile == 128 else s.t().contiguous()


def values(q, s, tile):
    q = q.double()
    per = s.double().t() if tile == 1 else s.double().repeat_interleave(128, 0)[:q.shape[0]]
    return q * per.repeat_interleave(128, 1)[:, :q.shape[1]]


def check8(q, s, y, tile, err):
    """q, s against y (float64), which the kernel had within `err`."""
    _, want = quant(y, tile)
    per = values(torch.ones_like(y), want, tile)
    emax = values(torch.ones_like(y), quant(err, tile)[1], tile) * 448   # the block's largest error
    assert ((values(torch.ones_like(y), s, tile) - per).abs() <= per * 2.0 ** -21 + emax / 448).all()
    got = values(q, s, tile)
    tol = torch.maximum(y.abs() * 2.0 ** -4, per * 2.0 ** -10) * 1.001 + 2 * err
    assert ((got - y).abs() <= tol).all()


def check(out, y, dtype, err):
    assert ((out.double() - y).abs() <= y.abs() * U[dtype] * 1.01 + err).all()


# ----------------------------------------------------------------------------
# root-mean-square norm
# ----------------------------------------------------------------------------

def rms(h, w, eps):
    y = h / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
    return y if w is None else y * w.double()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("rows,C,extra", [(1, 1, 0), (3, 8, 8), (5, 127, 1), (2, 129, 0), (1, 2048, 0), (333, 1000, 24),
                                          (700, 1152, 0), (9, 1160, 8), (40, 5120, 0), (3, 8200, 0), (2, 32768, 0),
                                          (4, 20001, 0), (1500, 64, 0)])
def test_rms_norm(cuda, dtype, q8, rows, C, extra):
    td, eps = TD[dtype], 1e-6
    x, r = held(rows, C, td, extra), held(rows, C, td, extra)
    x.copy_(randn((rows, C), 1, 2.0))
    r.copy_(randn((rows, C), 2, 3.0))
    w = (1 + randn((C,), 3, 0.3)).to(td)
    sm, out = held(rows, C, td, extra), held(rows, C, td, extra)
    q, s = held8(rows, C, 16), torch.empty((nb(C), rows), device=cuda)
    h = x.double() + r.double()
    y = rms(h, w, eps)
    ff.featfix_op_rms_norm(dtype, x, w, eps, resid=r, sum_out=sm, **({"q": q, "q_scale": s} if q8 else {"out": out}))
    torch.cuda.synchronize()
    check(sm, h, dtype, 0)
    err = y.abs() * (C + 8) * 2.0 ** -25 + y.abs() * 2.0 ** -21 + h.abs().amax() * 2.0 ** -24 * w.double().abs()
    if q8:
        check8(q, s, y, 1, err)
        assert untouched(q)
    else:
        check(out, y, dtype, err)
        assert untouched(out)
    assert untouched(sm) and untouched(x)


@pytest.mark.parametrize("C", [96, 1152, 9000])
def test_rms_norm_alone_in_place_and_unaligned(cuda, C):
    """No residual, no weight; then the sum over the residual itself; then rows
    that start off a 16-byte boundary."""
    x, r = randn((37, C), 4).bfloat16(), randn((37, C), 5).bfloat16()
    out = torch.empty_like(x)
    ff.featfix_op_rms_norm("bf16", x, None, 1e-5, out=out)
    y = rms(x.double(), None, 1e-5)
    check(out, y, "bf16", y.abs() * 1e-5)
    keep = r.clone()
    ff.featfix_op_rms_norm("bf16", x, None, 1e-5, resid=r, sum_out=r, out=out)
    h = x.double() + keep.double()
    check(r, h, "bf16", 0)
    first = out.clone()
    off = torch.zeros(37 * C + 1, device=cuda, dtype=torch.bfloat16)[1:].view(37, C)
    off.copy_(x)
    ff.featfix_op_rms_norm("bf16", off, None, 1e-5, resid=keep, sum_out=off, out=out)
    assert torch.equal(off, r)
    err = rms(h, None, 1e-5).abs() * (C * 2.0 ** -24)
    check(out, rms(h, None, 1e-5), "bf16", err)
    check(first, rms(h, None, 1e-5), "bf16", err)


def test_rms_norm_zero_and_special_rows(cuda):
    x = randn((6, 300), 6)
    x[0] = 0
    x[1, 200] = math.nan
    x[2, 5] = math.inf
    x[3] *= 1e-30
    q, s = held8(6, 300), torch.empty((3, 6), device=cuda)
    ff.featfix_op_rms_norm("f32", x, None, 1e-6, q=q, q_scale=s)
    v = values(q, s, 1)
    assert (v[0] == 0).all() and (s[:, 0] == 2.0 ** -100).all()
    assert torch.isnan(v[1]).all()             # the row's norm is NaN
    assert not torch.isfinite(v[2, 5]) and torch.isnan(v[2, 128:]).sum() == 0
    y = rms(x.double(), None, 1e-6)
    check8(q[3:], s[:, 3:].contiguous(), y[3:], 1, y[3:].abs() * 1e-5)


def test_rms_norm_offsets_past_32_bits(cuda):
    ld = (1 << 31) + 64
    big = torch.empty(2 * ld + 512, dtype=torch.bfloat16, device=cuda)
    x = torch.as_strided(big, (3, 256), (ld, 1))
    x.copy_(randn((3, 256), 7))
    q8 = torch.empty(2 * ld + 512, dtype=torch.uint8, device=cuda)
    q, s = torch.as_strided(q8, (3, 256), (ld, 1)).view(F8), torch.empty((2, 3), device=cuda)
    ff.featfix_op_rms_norm("bf16", x, None, 1e-6, q=q, q_scale=s)
    y = rms(x.double(), None, 1e-6)
    check8(q, s, y, 1, y.abs() * 1e-5)
    ff.featfix_op_quant8("bf16", x, q, s)
    check8(q, s, x.double(), 1, x.double() * 0)


# ----------------------------------------------------------------------------
# quantiser
# ----------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("rows,cols,extra", [(1, 1, 0), (1, 2048, 0), (127, 129, 8), (300, 1000, 3), (257, 96, 0),
                                             (1030, 1152, 0), (5, 8200, 8), (128, 128, 0)])
def test_quant8(cuda, dtype, tile, rows, cols, extra):
    x = held(rows, cols, TD[dtype], extra)
    x.copy_(randn((rows, cols), 8) * torch.exp(randn((1, cols), 9, 2.0)))
    q = held8(rows, cols, 16)
    s = torch.empty((nb(cols), rows) if tile == 1 else (nb(rows), nb(cols)), device=cuda)
    ff.featfix_op_quant8(dtype, x, q, s, tile)
    check8(q, s, x.double(), tile, x.double() * 0)
    assert untouched(q)


@pytest.mark.parametrize("tile", [1, 128])
def test_quant8_special_values(cuda, tile):
    x = randn((130, 400), 10)
    x[0, :128] = 0
    x[129] = 0
    x[2, 130] = math.nan
    x[3, 300] = -math.inf
    x[5] *= 1e-38
    q = held8(130, 400)
    s = torch.empty((4, 130) if tile == 1 else (2, 4), device=cuda)
    ff.featfix_op_quant8("f32", x, q, s, tile)
    v = values(q, s, tile)
    if tile == 1:
        assert (v[0, :128] == 0).all() and (v[129] == 0).all()
        assert torch.isnan(v[2, 128:256]).all() and torch.isfinite(v[2, :128]).all()
        assert torch.isnan(v[3, 256:384]).all() and torch.isfinite(v[3, 384:]).all()
        assert (v[5].abs() <= 2.0 ** -100).all()
    else:
        assert torch.isnan(v[:128, 128:384]).all() and torch.isfinite(v[:128, :128]).all()
        assert (v[129] == 0).all()


def test_quant8_keeps_representable_values(cuda):
    """Blocks of e4m3 values with 448 among them come back bit for bit."""
    codes = torch.arange(256, dtype=torch.uint8).cuda()
    codes = codes[(codes & 127) != 127]                       # all but the NaNs: 254 values
    x = codes.view(F8).float()[torch.randperm(254, generator=torch.Generator().manual_seed(0)).cuda()]
    x = torch.cat([x, x[:2]]).view(2, 128)
    x[:, 0] = 448
    q, s = held8(2, 128), torch.empty((1, 2), device=cuda)
    ff.featfix_op_quant8("f32", x, q, s)
    assert (s == 1).all() and torch.equal(q.float(), x)


# ----------------------------------------------------------------------------
# product
# ----------------------------------------------------------------------------

def gemm_inputs(M, N, K, seed, a_extra=0, w_extra=0):
    a, w = held8(M, K, a_extra), held8(N, K, w_extra)
    xa, xw = randn((M, K), seed) * torch.exp(randn((1, K), seed + 1)), randn((N, K), seed + 2, 0.05)
    qa, sa = quant(xa, 1)
    qw, sw = quant(xw, 128)
    a.copy_(qa)
    w.copy_(qw)
    return a, sa, w, sw


def gemm_ref(a, sa, w, sw):
    """(product, product of magnitudes) in float64."""
    A, W = values(a, sa, 1), values(w, sw, 128)
    return A @ W.t(), A.abs() @ W.abs().t()


def gelu64(x):
    return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))


SIZES = [(1, 8, 16), (1, 2048, 2048), (2, 130, 128), (7, 1000, 129), (16, 256, 4096), (17, 100, 1000), (33, 520, 640),
         (64, 384, 96), (100, 2048, 8192), (128, 128, 128), (129, 129, 257), (200, 72, 1), (256, 2048, 512),
         (300, 1152, 1160), (500, 1000, 712), (1000, 4608, 256), (1027, 1031, 1040), (2049, 640, 384), (4100, 1152, 300),
         (6000, 2050, 200)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_gemm8(cuda, dtype, M, N, K):
    td = TD[dtype]
    a, sa, w, sw = gemm_inputs(M, N, K, 20, 16, 32)
    ref, mag = gemm_ref(a, sa, w, sw)
    # 128 products to a block, then a sum over the blocks, and the scales' product
    err = mag * (128 + nb(K) + 4) * 2.0 ** -24
    bias = randn((N,), 23).to(td)
    out = held(M, N, td)
    ff.featfix_op_gemm8(dtype, a, sa, w, sw, out=out)
    check(out, ref, dtype, err)
    y = ref + bias.double()
    ff.featfix_op_gemm8(dtype, a, sa, w, sw, out=out, bias=bias)
    check(out, y, dtype, err + y.abs() * 2.0 ** -24)
    # |GELU'| <= 1.13, and the GELU itself within a few fp32 roundings of its argument
    g = gelu64(y)
    gerr = 1.13 * err + y.abs() * 2.0 ** -20
    ff.featfix_op_gemm8(dtype, a, sa, w, sw, out=out, bias=bias, act=1)
    check(out, g, dtype, gerr)
    q, s = held8(M, N, 16), torch.empty((nb(N), M), device=cuda)
    ff.featfix_op_gemm8(dtype, a, sa, w, sw, bias=bias, act=1, q=q, q_scale=s)
    check8(q, s, g, 1, gerr)
    assert untouched(q)
    ff.featfix_op_gemm8(dtype, a, sa, w, sw, q=q, q_scale=s)
    check8(q, s, ref, 1, err)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K,rpb", [(1, 130, 256, 1), (5, 1000, 300, 2), (70, 512, 128, 7), (300, 1152, 512, 256),
                                       (1030, 1032, 256, 40), (2050, 2304, 384, 1000),
                                       (3100, 1537, 200, 300), (2600, 2050, 130, 9)])
@pytest.mark.parametrize("extra", [0, 5, 8])
def test_gemm8_gate_and_residual(cuda, dtype, M, N, K, rpb, extra):
    td = TD[dtype]
    a, sa, w, sw = gemm_inputs(M, N, K, 30)
    ref, mag = gemm_ref(a, sa, w, sw)
    err = mag * (128 + nb(K) + 4) * 2.0 ** -24
    bias = randn((N,), 33).to(td)
    gate = randn((-(-M // rpb), 2 * N + 3), 34)[:, N:2 * N]
    resid, out = held(M, N, td, extra), held(M, N, td, extra)
    resid.copy_(randn((M, N), 35, 2.0))
    y = ref + bias.double()
    gm = gate.double().repeat_interleave(rpb, 0)[:M]
    want = resid.double() + gm * y
    terr = gm.abs() * (err + y.abs() * 2.0 ** -23) + want.abs() * 2.0 ** -23
    ff.featfix_op_gemm8(dtype, a, sa, w, sw, out=out, bias=bias, gate=gate, rows_per_batch=rpb, resid=resid)
    check(out, want, dtype, terr)
    assert untouched(out)
    ff.featfix_op_gemm8(dtype, a, sa, w, sw, out=out, bias=bias, resid=resid)
    check(out, resid.double() + y, dtype, err + (resid.double().abs() + y.abs()) * 2.0 ** -23)
    ff.featfix_op_gemm8(dtype, a, sa, w, sw, out=resid, bias=bias, gate=gate, rows_per_batch=rpb, resid=resid)
    check(resid, want, dtype, terr)
    assert untouched(resid)


@pytest.mark.parametrize("M,N,K", [(1, 2048, 2048), (130, 700, 384), (3000, 2304, 512)])
def test_gemm8_repeats_itself(cuda, M, N, K):
    """Sums in a fixed order: the same bits every time, on another stream too."""
    a, sa, w, sw = gemm_inputs(M, N, K, 40)
    outs = [held(M, N, torch.float32) for _ in range(6)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for i, o in enumerate(outs):
        if i % 2:
            with torch.cuda.stream(side):
                ff.featfix_op_gemm8("f32", a, sa, w, sw, out=o)
        else:
            ff.featfix_op_gemm8("f32", a, sa, w, sw, out=o)
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert torch.equal(o, outs[0])


@pytest.mark.parametrize("M,N", [(3, 300), (700, 520), (5000, 2304)])
def test_gemm8_special_values_stay_in_their_rows(cuda, M, N):
    """A NaN row of A (or an infinite scale) and a NaN block of W reach their own
    rows and columns of the product, and no other."""
    K = 384
    a, sa, w, sw = gemm_inputs(M, N, K, 50)
    sa, sw = sa.clone(), sw.clone()
    sa[1, 1] = math.nan
    sa[2, 2] = math.inf
    sw[1, 0] = math.nan
    out = held(M, N, torch.float32)
    ff.featfix_op_gemm8("f32", a, sa, w, sw, out=out)
    bad = ~torch.isfinite(out)
    want = torch.zeros_like(bad)
    want[1:3] = True
    want[:, 128:256] = True
    assert torch.equal(bad, want)


def test_gemm8_offsets_past_32_bits(cuda):
    """A, the residual and the output with row strides that pass 2^32 bytes."""
    M, N, K, ld = 140, 200, 256, 1 << 25
    a, sa, w, sw = gemm_inputs(M, N, K, 60)
    far = torch.empty((M - 1) * ld + K, dtype=torch.uint8, device=cuda)
    A = torch.as_strided(far, (M, K), (ld, 1)).view(F8)
    A.copy_(a)
    fo = torch.empty((M - 1) * ld + N, dtype=torch.bfloat16, device=cuda)
    out = torch.as_strided(fo, (M, N), (ld, 1))
    r = randn((M, N), 61).bfloat16()
    out.copy_(r)
    ref, mag = gemm_ref(a, sa, w, sw)
    ff.featfix_op_gemm8("bf16", A, sa, w, sw, out=out, resid=out)
    check(out, ref + r.double(), "bf16", mag * 2.0 ** -16 + (ref.abs() + r.double().abs()) * 2.0 ** -23)


@pytest.mark.parametrize("M", [4, 300, 3000])
def test_gemm8_watchdog_is_quiet(cuda, M):
    a, sa, w, sw = gemm_inputs(M, 300, 700, 63)
    ff.featfix_op_gemm8("f32", a, sa, w, sw, out=held(M, 300, torch.float32))
    ff.featfix_op_gemm8_watchdog()


# ----------------------------------------------------------------------------
# rotary positions
# ----------------------------------------------------------------------------

def rope_ref(x, pos, axes, hd, theta, halves, ladder, inverse, weight, eps):
    rows, rot = x.shape[0], sum(axes)
    v = x.double().view(rows, -1, hd).clone()
    if weight is not None:
        v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + eps) * weight.double()
    y, p = v.clone(), 0
    for a, width in enumerate(axes):
        for i in range(width // 2):
            f = theta ** (-2 * p / rot) if ladder else theta ** (-2 * i / width)
            ang = (pos[a].double() * f * (-1 if inverse else 1))[:, None]
            j, k = (p, p + rot // 2) if halves else (2 * p, 2 * p + 1)
            y[..., j] = v[..., j] * ang.cos() - v[..., k] * ang.sin()
            y[..., k] = v[..., j] * ang.sin() + v[..., k] * ang.cos()
            p += 1
    return y.view(rows, -1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("rows,hq,hk,hd,axes,ladder,extra", [
    (1, 1, 1, 2, (2,), False, 0), (1, 16, 4, 128, (32, 48, 48), True, 0), (5, 3, 1, 32, (8, 12, 12), False, 1),
    (300, 4, 4, 72, (24, 24, 24), False, 8), (33, 2, 1, 80, (20, 30), True, 0), (17, 6, 2, 96, (96,), False, 0),
    (260, 8, 8, 128, (16, 56, 56), False, 0), (9, 5, 5, 256, (64, 64, 64, 64), False, 3), (40, 2, 2, 50, (6, 10, 14), False, 0),
    (2100, 16, 16, 64, (16, 24, 24), False, 0), (70, 3, 0, 128, (64,), True, 8), (3, 40, 10, 66, (66,), False, 0),
    (4, 1, 1, 16, (2, 2, 2, 2, 2, 2, 2, 2), False, 0),
    (1300, 6, 2, 128, (54, 20), True, 8), (45, 3, 1, 40, (14, 8), False, 0),
    (20, 3, 1, 256, (200, 54), False, 0), (700, 5, 3, 72, (10, 20, 16), True, 1), (9, 2, 2, 34, (6, 12), False, 2)])
def test_rope(cuda, dtype, halves, norm, rows, hq, hk, hd, axes, ladder, extra):
    td, theta, eps = TD[dtype], 10000.0, 1e-6
    qkv = randn((rows, (hq + 2 * hk) * hd + extra), 70).to(td)
    q, k = qkv[:, :hq * hd], qkv[:, hq * hd:(hq + hk) * hd]
    g = torch.Generator().manual_seed(71)
    pos = torch.randint(-50, 40000, (len(axes), rows), generator=g, dtype=torch.int32).cuda()
    wq, wk = ((1 + randn((hd,), 72, 0.3)).to(td), (1 + randn((hd,), 73, 0.3)).to(td)) if norm else (None, None)
    qo, ko = held(rows, hq * hd, td, extra), held(rows, hk * hd, td, extra) if hk else None
    kw = dict(theta=theta, halves=halves, one_ladder=ladder, q_weight=wq, eps=eps)
    if hk:
        kw.update(k=k, k_out=ko, k_weight=wk)
    ff.featfix_op_rope(dtype, pos, axes, hd, q=q, q_out=qo, **kw)
    for x, o, w in ((q, qo, wq), (k, ko, wk))[:2 if hk else 1]:
        want = rope_ref(x, pos, axes, hd, theta, halves, ladder, False, w, eps)
        # cos and sin within a few fp32 roundings (angle included) of a pair of at most 8
        assert ((o.double() - want).abs() <= want.abs() * U[dtype] * 1.01 + 8 * 2.0 ** -21).all()
        assert untouched(o)
    # in place
    keep = qkv.clone()
    if hk:
        kw["k_out"] = k
    ff.featfix_op_rope(dtype, pos, axes, hd, q=q, q_out=q, **kw)
    assert torch.equal(q, qo) and (not hk or torch.equal(k, ko))
    assert torch.equal(qkv[:, (hq + hk) * hd:], keep[:, (hq + hk) * hd:])


@pytest.mark.parametrize("halves", [False, True])
def test_rope_inverse_is_the_gradient(cuda, halves):
    """The rotation is linear and orthogonal: its gradient is the inverse.  Against
    differences of <g, rope(x)> (exact for a linear map, up to rounding) and the
    round trip."""
    rows, H, hd, axes = 12, 3, 48, (8, 20, 12)
    x, g = randn((rows, H * hd), 74), randn((rows, H * hd), 75)
    pos = torch.randint(0, 500, (3, rows), generator=torch.Generator().manual_seed(76), dtype=torch.int32).cuda()

    def rope(v, inverse=False):
        o = torch.empty_like(v)
        ff.featfix_op_rope("f32", pos, axes, hd, q=v, q_out=o, halves=halves, inverse=inverse)
        return o

    grad = rope(g, True)
    assert ((rope(rope(x), True) - x).abs() <= 8 * 2.0 ** -20).all()
    for seed in range(4):
        d = randn((rows, H * hd), 80 + seed)
        diff = (g.double() * (rope(x + d).double() - rope(x - d).double())).sum() / 2
        want = (grad.double() * d.double()).sum()
        assert abs(diff - want) <= 64 * 2.0 ** -22 * math.sqrt(rows * H * hd) * 8
    ref = rope_ref(g, pos, axes, hd, 10000.0, halves, False, True, None, 0)
    assert ((grad.double() - ref).abs() <= 8 * 2.0 ** -21).all()


@pytest.mark.parametrize("first", [0, 1 << 20, 123456789, 2 ** 31 - 40, -2 ** 31])
def test_rope_positions_of_every_size(cuda, first):
    pos = (first + torch.arange(32, dtype=torch.int64)).to(torch.int32).cuda()[None]
    x = torch.ones((32, 128), device=cuda)
    o = torch.empty_like(x)
    ff.featfix_op_rope("f32", pos, (128,), 128, q=x, q_out=o)
    want = rope_ref(x, pos, (128,), 128, 10000.0, False, False, False, None, 0)
    assert (o.double() - want).abs().max() <= (2.0 ** -20 if abs(first) <= 1 << 20 else 6e-5)


def test_rope_offsets_past_32_bits(cuda):
    ld = (1 << 31) + 8
    big = torch.empty(2 * ld + 512, dtype=torch.bfloat16, device=cuda)
    x = torch.as_strided(big, (3, 256), (ld, 1))
    x.copy_(randn((3, 256), 90))
    keep = x.clone()
    pos = torch.tensor([[5, 6, 7]], dtype=torch.int32, device=cuda)
    ff.featfix_op_rope("bf16", pos, (128,), 128, q=x, q_out=x)
    want = rope_ref(keep, pos, (128,), 128, 10000.0, False, False, False, None, 0)
    assert ((x.double() - want).abs() <= want.abs() * 2.0 ** -8 * 1.01 + 2.0 ** -18).all()


# ----------------------------------------------------------------------------
# empty calls
# ----------------------------------------------------------------------------

def test_no_rows_do_nothing(cuda):
    n0 = ff.featfix_launch_count()
    x, q, s = torch.empty((0, 256), dtype=torch.bfloat16, device=cuda), held8(1, 256)[:0], torch.empty((2, 0), device=cuda)
    ff.featfix_op_rms_norm("bf16", x, None, 1e-6, out=x)
    ff.featfix_op_rms_norm("bf16", x, None, 1e-6, q=q, q_scale=s)
    ff.featfix_op_quant8("bf16", x, q, s)
    ff.featfix_op_quant8("bf16", x, q, torch.empty((0, 2), device=cuda), tile=128)
    w, sw = quant(randn((256, 256), 91), 128)
    ff.featfix_op_gemm8("bf16", q, s, w, sw, out=x)
    ff.featfix_op_rope("bf16", torch.empty((1, 0), dtype=torch.int32, device=cuda), (128,), 128, q=x, q_out=x)
    assert ff.featfix_launch_count() == n0
