"""Every stage of the 8-bit block (block8.Block8) against its formula in float64,
from what the stage before it left in the block's buffers.

The block's arithmetic is followed call by call: after each operator the buffers are
copied, and the next stage's result is computed from these copies and the block's own
weights, so that only that stage's roundings separate the two.  Bounds: those of the
operators' own tests (test_gpu_ops8.py), the attention's those of its tests (a relative
error of 1e-2).  Stages computed with a step left out or exchanged must lie outside them."""

import math

import pytest
import torch

from paper_2607_27842_gb300 import block8

from .test_gpu_block8 import weights
from .test_gpu_ops8 import check, check8, gelu64, nb, rms, rope_ref, values

pytestmark = pytest.mark.gpu

EPS = 1e-6
CASES = [(1, 5, 1, 4, 4, 2, 64, (16, 24, 24)), (2, 17, 2, 6, 7, 4, 64, (16, 24, 24)), (1, 32, 3, 9, 11, 4, 128, (16, 56, 56)),
         (2, 0, 1, 16, 16, 8, 72, (24, 24, 24)), (1, 256, 2, 15, 20, 6, 128, (16, 56, 56))]
NAMES = ["rms_norm", "gemm8", "rope", "attention", "quant8", "gemm8", "rms_norm", "gemm8", "gemm8"]


def stages(monkeypatch, blk, x, pos):
    """Copies of the buffers before the block and after each of its operators."""
    got, names = [], []

    def copy():
        got.append({"x": x.clone(), "qkv": blk.qkv.clone(), "o": blk.o.clone(), "d": blk.d.clone(),
                    "a": tuple(t.clone() for t in blk.a), "h": tuple(t.clone() for t in blk.h)})

    def follow(name):
        op = getattr(block8.ff, "featfix_op_" + name)

        def call(*args, **kw):
            op(*args, **kw)
            names.append(name)
            copy()
        monkeypatch.setattr(block8.ff, "featfix_op_" + name, call)

    for name in sorted(set(NAMES)):
        follow(name)
    copy()
    blk(x, pos)
    torch.cuda.synchronize()
    assert names == NAMES
    return got


def eight(t):
    """The values of an 8-bit activation and its scales."""
    return values(t[0].view(torch.float8_e4m3fn), t[1], 1)


def product(a, w8, bias):
    """a W^T + bias in float64 and the bound of its fp32 error."""
    A, W = eight(a), values(w8[0].view(torch.float8_e4m3fn), w8[1], 128)
    y = A @ W.t() + bias.double()
    return y, A.abs() @ W.abs().t() * (128 + nb(A.shape[1]) + 4) * 2.0 ** -24 + y.abs() * 2.0 ** -24


def attended(qkv, heads, dim, batch, n_txt, n_img):
    C = heads * dim
    q, k, v = (qkv[:, i * C:(i + 1) * C].double().view(-1, heads, dim) for i in range(3))
    o = torch.empty_like(q)
    for b in range(batch):
        rows = torch.cat([torch.arange(n_txt) + b * n_txt, batch * n_txt + b * n_img + torch.arange(n_img)]).to(q.device)
        p = torch.softmax(torch.einsum("nhd,mhd->hnm", q[rows], k[rows]) / math.sqrt(dim), -1)
        o[rows] = torch.einsum("hnm,mhd->nhd", p, v[rows])
    return o.reshape(-1, C)


def norm_err(h, y, w):
    C = h.shape[1]
    return y.abs() * ((C + 8) * 2.0 ** -25 + 2.0 ** -21) + h.abs().amax() * 2.0 ** -24 * w.double().abs()


def outside(f, *args):
    """The check does not pass."""
    with pytest.raises(AssertionError):
        f(*args)


@pytest.mark.parametrize("batch,n_txt,frames,height,width,heads,dim,axes", CASES)
def test_block8_stage_by_stage(cuda, monkeypatch, batch, n_txt, frames, height, width, heads, dim, axes):
    C, n_img = heads * dim, frames * height * width
    w = weights(C, 4 * C, dim, 5)
    # attention weights far from uniform: what it reads of q and k shows
    w["q_norm"], w["k_norm"] = w["q_norm"] * 2, w["k_norm"] * 2
    pos = block8.joint_positions(batch, n_txt, frames, height, width)
    blk = block8.Block8(w, heads, axes, batch, n_txt, n_img)
    x0 = (torch.randn((blk.rows, C), generator=torch.Generator().manual_seed(6)) * 1.5).bfloat16().cuda()
    s = stages(monkeypatch, blk, x0, pos)
    f8 = torch.float8_e4m3fn

    def is8(t, y, err):
        check8(t[0].view(f8), t[1], y, 1, err)

    for m in block8.MATRICES:
        W = w[m + ".w"].double()
        check8(blk.q8[m][0].view(f8), blk.q8[m][1], W, 128, W * 0)

    # norm in front of the attention
    h = s[0]["x"].double()
    y = rms(h, w["norm1"], EPS)
    is8(s[1]["a"], y, norm_err(h, y, w["norm1"]))
    outside(is8, s[1]["a"], rms(h, w["norm2"], EPS), norm_err(h, y, w["norm1"]))
    # q, k, v
    y, err = product(s[1]["a"], blk.q8["qkv"], w["qkv.b"])
    check(s[2]["qkv"], y, "bf16", err)
    outside(check, s[2]["qkv"], y - w["qkv.b"].double(), "bf16", err)
    # rotary positions on the normalised q and k, v as it was
    before, after = s[2]["qkv"], s[3]["qkv"]
    assert torch.equal(after[:, 2 * C:], before[:, 2 * C:])
    for i, name in enumerate(("q_norm", "k_norm")):
        part, got = before[:, i * C:(i + 1) * C], after[:, i * C:(i + 1) * C]
        turn = lambda p, g, ax: rope_ref(part, p, ax, dim, 10000.0, False, False, False, g, EPS)
        near = lambda want: check(got, want, "bf16", 24 * 2.0 ** -21)   # (normalised values times weights: at most 24)
        near(turn(pos, w[name], axes))
        outside(near, turn(pos * 0, w[name], axes))                    # no rotation
        outside(near, turn(pos.flip(0), w[name], axes))                # the axes in another order
        outside(near, turn(pos, torch.ones_like(w[name]), axes))       # no weight
        outside(near, turn(pos, w["k_norm" if i == 0 else "q_norm"], axes))
    # attention
    want = attended(after, heads, dim, batch, n_txt, n_img)
    off = lambda t: float((s[4]["o"].double() - t).norm() / t.norm())
    assert off(want) < 1e-2
    assert off(attended(before, heads, dim, batch, n_txt, n_img)) > 1e-2
    assert off(after[:, 2 * C:].double()) > 1e-2
    # its output in 8 bits, the out-projection
    is8(s[5]["a"], s[4]["o"].double(), want * 0)
    y, err = product(s[5]["a"], blk.q8["proj"], w["proj.b"])
    check(s[6]["d"], y, "bf16", err)
    outside(check, s[6]["d"], y - w["proj.b"].double(), "bf16", err)
    # residual, norm in front of the MLP
    assert torch.equal(s[6]["x"], s[0]["x"])
    h = s[0]["x"].double() + s[6]["d"].double()
    check(s[7]["x"], h, "bf16", 0)
    y = rms(h, w["norm2"], EPS)
    is8(s[7]["a"], y, norm_err(h, y, w["norm2"]))
    outside(is8, s[7]["a"], rms(h, None, EPS), norm_err(h, y, w["norm2"]))
    outside(is8, s[7]["a"], rms(s[0]["x"].double(), w["norm2"], EPS), norm_err(h, y, w["norm2"]))
    # the MLP
    y, err = product(s[7]["a"], blk.q8["fc1"], w["fc1.b"])
    is8(s[8]["h"], gelu64(y), 1.13 * err + y.abs() * 2.0 ** -20)
    outside(is8, s[8]["h"], y, 1.13 * err + y.abs() * 2.0 ** -20)
    y, err = product(s[8]["h"], blk.q8["fc2"], w["fc2.b"])
    y, r = y + s[7]["x"].double(), s[7]["x"].double()
    err = err + (r.abs() + y.abs()) * 2.0 ** -23
    check(s[9]["x"], y, "bf16", err)
    outside(check, s[9]["x"], y - w["fc2.b"].double(), "bf16", err)
    outside(check, s[9]["x"], y - r, "bf16", err)
