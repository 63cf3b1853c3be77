"""Refusals of the 8-bit layer operators: every argument is checked on the host
before anything is launched (no GPU needed)."""

import ctypes
import math
import os

import pytest
import torch

from paper_2607_27842_gb300 import featfix as ff

P = 1 << 20      # an address that is never read: the calls are refused before
NULL = None


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ff.LIB_PATH):
        from paper_2607_27842_gb300 import build
        build.build()
    return ff.lib()


RMS = dict(dtype=1, rows=4, C=256, x=P, ldx=256, resid=P, ldr=256, sum=P, ldsum=256, weight=P, eps=1e-6, out=NULL, ldo=0,
           q=P, ldq=256, scale=P, lds=4, stream=NULL)
QUANT = dict(dtype=0, tile=1, rows=4, cols=200, x=P, ldx=200, q=P, ldq=208, scale=P, lds=4, stream=NULL)
GEMM = dict(dtype=1, M=4, N=200, K=300, a=P, lda=304, sa=P, ldsa=4, w=P, ldw=304, sw=P, ldsw=3, bias=P, act=0, gate=P,
            gs=200, rpb=4, resid=P, ldr=200, out=P, ldo=200, q=NULL, ldq=0, qs=NULL, ldqs=0, stream=NULL)
ROPE = dict(dtype=1, rows=4, hd=64, n_axes=2, axes=(32, 32), pos=P, ldp=4, theta=1e4, flags=0, q=P, ldq=256, hq=4, wq=NULL,
            qo=P, ldqo=256, k=P, ldk=128, hk=2, wk=NULL, ko=P, ldko=128, eps=1e-6, stream=NULL)


def call(lib, name, args):
    a = dict(args)
    if "axes" in a and a["axes"] is not None:
        a["axes"] = (ctypes.c_int * len(a["axes"]))(*a["axes"])
    return getattr(lib, name)(*a.values())


BAD = [("featfix_op_rms_norm", RMS, b) for b in (
    dict(dtype=2), dict(rows=-1), dict(rows=1 << 31), dict(C=0), dict(C=32769, ldx=40000, ldr=40000, ldsum=40000, ldq=40000),
    dict(x=NULL), dict(ldx=255), dict(x=P + 1), dict(ldr=255), dict(resid=P + 1), dict(ldsum=128), dict(weight=P + 1),
    dict(eps=-1.0), dict(eps=math.nan), dict(q=NULL), dict(out=P, ldo=256), dict(scale=NULL), dict(ldq=264), dict(ldq=240),
    dict(q=P + 8), dict(lds=3), dict(scale=P + 2), dict(q=NULL, out=P, ldo=255), dict(q=NULL, out=P + 1, ldo=256))]
BAD += [("featfix_op_quant8", QUANT, b) for b in (
    dict(dtype=-1), dict(tile=0), dict(tile=64), dict(rows=-1), dict(cols=0), dict(x=NULL), dict(x=P + 2), dict(ldx=199),
    dict(q=NULL), dict(q=P + 4), dict(ldq=200), dict(ldq=192), dict(scale=NULL), dict(lds=3), dict(tile=128, lds=1))]
BAD += [("featfix_op_gemm8", GEMM, b) for b in (
    dict(dtype=5), dict(M=-1), dict(N=0), dict(K=0), dict(a=NULL), dict(a=P + 8), dict(lda=300), dict(lda=288), dict(sa=NULL),
    dict(ldsa=3), dict(w=NULL), dict(ldw=301), dict(sw=NULL), dict(sw=P + 1), dict(ldsw=2), dict(bias=P + 1), dict(act=2),
    dict(rpb=0), dict(gs=199), dict(gate=P + 2), dict(ldr=199), dict(resid=P + 1), dict(out=NULL), dict(ldo=199),
    dict(q=P, ldq=208, qs=P, ldqs=4), dict(out=NULL, q=P, ldq=208, qs=P, ldqs=4),
    dict(out=NULL, gate=NULL, resid=NULL, q=P, ldq=200, qs=P, ldqs=4),
    dict(out=NULL, gate=NULL, resid=NULL, q=P, ldq=208, qs=NULL, ldqs=4),
    dict(out=NULL, gate=NULL, resid=NULL, q=P, ldq=208, qs=P, ldqs=3))]
BIG = (1 << 31) - 255
BAD += [("featfix_op_gemm8", GEMM, b) for b in (dict(M=BIG, ldsa=1 << 31), dict(N=BIG, gs=1 << 31, ldr=1 << 31, ldo=1 << 31),
                                               dict(K=BIG, lda=1 << 31, ldw=1 << 31, ldsw=1 << 25))]
BAD += [("featfix_op_quant8", QUANT, dict(cols=BIG, ldx=1 << 31, ldq=1 << 31)),
        ("featfix_op_rope", ROPE, dict(hq=65530, hd=2, axes=(2,), n_axes=1, ldq=1 << 20, ldqo=1 << 20, hk=6))]
BAD += [("featfix_op_rope", ROPE, b) for b in (
    dict(dtype=3), dict(rows=-1), dict(hd=63), dict(hd=0), dict(hd=258, ldq=2000, ldqo=2000, ldk=2000, ldko=2000),
    dict(n_axes=0), dict(n_axes=9), dict(axes=None), dict(axes=(32, 34)), dict(axes=(31, 33)), dict(axes=(0, 64)),
    dict(axes=(-2, 64)), dict(pos=NULL), dict(pos=P + 2), dict(ldp=3), dict(theta=0.0), dict(theta=-1.0),
    dict(theta=math.nan), dict(theta=math.inf), dict(flags=8), dict(q=NULL), dict(ldq=255), dict(q=P + 1), dict(qo=NULL),
    dict(ldqo=255), dict(hq=-1), dict(hq=0, hk=0), dict(ko=NULL), dict(ldk=127), dict(ldko=127), dict(eps=-1.0),
    dict(wq=P, flags=4), dict(wk=P, flags=4), dict(wq=P + 1), dict(hq=1 << 30, ldq=1 << 40, ldqo=1 << 40))]


@pytest.mark.parametrize("name,good,bad", BAD, ids=["%s-%s" % (n[11:], "-".join(map(str, b))) for n, _, b in BAD])
def test_refused(lib, name, good, bad):
    assert set(bad) <= set(good)
    n0 = ff.featfix_launch_count()
    assert call(lib, name, {**good, **bad}) == ff.ERR_INVALID_ARG
    assert ff.featfix_launch_count() == n0


@pytest.mark.parametrize("name,good,none", [
    ("featfix_op_rms_norm", RMS, dict(rows=0)), ("featfix_op_quant8", QUANT, dict(rows=0)),
    ("featfix_op_quant8", QUANT, dict(rows=0, tile=128, lds=2)), ("featfix_op_gemm8", GEMM, dict(M=0)),
    ("featfix_op_rope", ROPE, dict(rows=0))])
def test_no_rows_are_accepted_and_launch_nothing(lib, name, good, none):
    """(the unchanged arguments pass every check: what test_refused changes is what is refused)"""
    n0 = ff.featfix_launch_count()
    assert call(lib, name, {**good, **none}) == ff.OK
    assert ff.featfix_launch_count() == n0


def test_binding_refuses_wrong_tensors():
    f8 = torch.float8_e4m3fn
    x = torch.zeros((4, 256), dtype=torch.bfloat16)
    q, s = torch.zeros((4, 256), dtype=torch.uint8).view(f8), torch.zeros((2, 4))
    bad = [lambda: ff.featfix_op_rms_norm("bf16", x, None, 1e-6, q=q, q_scale=s),               # not on a GPU
           lambda: ff.featfix_op_rms_norm("f32", x, None, 1e-6, out=x),                         # type
           lambda: ff.featfix_op_rms_norm("bf16", x[0], None, 1e-6, out=x),                     # dimensions
           lambda: ff.featfix_op_rms_norm("bf16", x.t(), None, 1e-6, out=x),                    # order
           lambda: ff.featfix_op_quant8("bf16", x, q, torch.zeros((4, 2))),                     # scales the other way
           lambda: ff.featfix_op_quant8("bf16", x, q, None),
           lambda: ff.featfix_op_quant8("bf16", x, q, s, tile=128),
           lambda: ff.featfix_op_gemm8("bf16", q, s, q[:, :128], torch.zeros((1, 2)), out=x),   # K of A and W
           lambda: ff.featfix_op_rope("bf16", torch.zeros((1, 4), dtype=torch.int32), (96,), 96, q=x, q_out=x)]
    for b in bad:
        with pytest.raises(ff.FeatFixError) as e:
            b()
        assert e.value.status == ff.ERR_INVALID_ARG
