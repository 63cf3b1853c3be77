"""Refusals of the 8-bit key-value cache's operators and of the block norms: every
argument is checked on the host before anything is launched (no GPU needed)."""

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


CACHE = dict(k=P, v=P, k_scale=P, v_scale=P, k_stride=(4096, 256, 80), v_stride=(4096, 256, 80), k_scale_stride=(48, 3, 1),
             v_scale_stride=(48, 1, 16), pages=8, page_size=16, heads=3, head_dim=72, table=P, ld_table=5, table_pages=5, seqs=4,
             lens=P)
ROWS = dict(dtype=1, cache=CACHE, rows=7, row_start=P, k=P, ldk=216, v=P, ldv=216, stream=NULL)
ATTN = dict(dtype=0, cache=CACHE, q=P, ldq=432, heads=6, scale=0.1, window=0, out=P, ldo=432, lse=P, ws=P, bytes=1 << 34,
            stream=NULL)
NORMS = dict(dtype=1, rows=9, C=200, flags=3, eps=1e-6, y=P, ldy=200, wa=P, gate=P, gs=200, x=P, ldx=200, rs=0.5, sum=P, ldsum=200,
             w=P, scale=P, ss=200, shift=P, shs=200, rpb=4, out=NULL, ldo=0, q=P, ldq=208, qs=P, ldqs=9, stream=NULL)


def call(lib, name, args):
    a = dict(args)
    if "cache" in a and a["cache"] is not None:
        c = ff.KvCache()
        for n, v in a["cache"].items():
            setattr(c, n, (ctypes.c_longlong * 3)(*v) if isinstance(v, tuple) else v)
        a["cache"] = ctypes.byref(c)
    return getattr(lib, name)(*a.values())


BAD_CACHE = [
    dict(k=NULL), dict(v=NULL), dict(k=P + 8), dict(v=P + 1), dict(k_scale=NULL), dict(v_scale=P + 2), dict(table=NULL),
    dict(table=P + 2), dict(lens=NULL), dict(lens=P + 1), dict(k_stride=(4096, 256, 72)), dict(v_stride=(4096, 256, 64)),
    dict(k_stride=(4096, 40, 80)), dict(k_stride=(0, 256, 80)), dict(v_stride=(-4096, 256, 80)), dict(v_stride=(1 << 60, 256, 80)),
    dict(k_scale_stride=(48, 0, 1)), dict(v_scale_stride=(48, 3, -1)), dict(pages=0), dict(pages=-1), dict(page_size=0),
    dict(page_size=(1 << 24) + 1), dict(heads=0), dict(heads=65536), dict(head_dim=0), dict(head_dim=12), dict(head_dim=-8),
    dict(head_dim=264), dict(table_pages=0), dict(table_pages=1 << 27, ld_table=1 << 27), dict(ld_table=4), dict(seqs=-1)]
BAD = [(n, g, dict(cache={**CACHE, **b})) for b in BAD_CACHE
       for n, g in (("featfix_op_kv_write", ROWS), ("featfix_op_kv_attention", ATTN))]
BAD += [(n, ROWS, b) for n in ("featfix_op_kv_write", "featfix_op_kv_read") for b in (
    dict(dtype=2), dict(cache=NULL), dict(rows=-1), dict(rows=1 << 31), dict(row_start=NULL), dict(row_start=P + 2), dict(k=NULL),
    dict(k=P + 1), dict(ldk=215), dict(v=NULL), dict(v=P + 1), dict(ldv=215))]
BAD += [("featfix_op_kv_attention", ATTN, b) for b in (
    dict(dtype=-1), dict(cache=NULL), dict(q=NULL), dict(q=P + 2), dict(ldq=431), dict(heads=0), dict(heads=7), dict(heads=-3),
    dict(heads=65538), dict(scale=math.nan), dict(scale=math.inf), dict(window=-1), dict(out=NULL), dict(out=P + 2), dict(ldo=431),
    dict(lse=P + 2))]
BAD += [("featfix_op_block_norms", NORMS, b) for b in (
    dict(dtype=7), dict(rows=-1), dict(rows=1 << 31), dict(C=0), dict(C=16385, ldy=20000, ldx=20000, ldsum=20000, ldq=20000,
    gs=20000, ss=20000, shs=20000), dict(flags=4), dict(flags=2), dict(eps=-1.0), dict(eps=math.nan), dict(y=NULL), dict(y=P + 1),
    dict(ldy=199), dict(wa=P + 1), dict(gate=P + 2), dict(gs=199), dict(x=P + 1), dict(ldx=199), dict(rs=math.nan), dict(rs=math.inf),
    dict(sum=P + 1), dict(ldsum=199), dict(w=P + 1), dict(scale=P + 1), dict(ss=0), dict(shift=P + 3), dict(shs=-200), dict(rpb=0),
    dict(out=P, ldo=200), dict(q=NULL, out=P, ldo=199), dict(q=NULL, out=P + 1, ldo=200), dict(q=NULL, sum=NULL), dict(q=P + 8),
    dict(ldq=200), dict(ldq=192), dict(qs=NULL), dict(qs=P + 2), dict(ldqs=8))]


@pytest.mark.parametrize("name,good,bad", BAD, ids=["%s-%d" % (n[11:], i) for i, (n, _, _) in enumerate(BAD)])
def test_refused(lib, name, good, bad):
    assert set(bad) <= set(good)
    n0 = ff.featfix_launch_count()
    assert call(lib, name, {**good, **bad}) == ff.ERR_INVALID_ARG
    assert ff.featfix_launch_count() == n0


EMPTY = {**CACHE, "seqs": 0}


@pytest.mark.parametrize("name,good,none", [
    ("featfix_op_kv_write", ROWS, dict(rows=0)), ("featfix_op_kv_read", ROWS, dict(rows=0)),
    ("featfix_op_kv_write", ROWS, dict(cache=EMPTY)), ("featfix_op_kv_read", ROWS, dict(cache=EMPTY, rows=0, row_start=NULL)),
    ("featfix_op_kv_attention", ATTN, dict(cache=EMPTY)), ("featfix_op_block_norms", NORMS, dict(rows=0))])
def test_no_rows_are_accepted_and_launch_nothing(lib, name, good, none):
    n0 = ff.featfix_launch_count()
    assert call(lib, name, {**good, **none}) == ff.OK
    assert ff.featfix_launch_count() == n0


@pytest.mark.parametrize("seqs,q_heads,heads,dim,tokens", [(1, 16, 4, 128, 131072), (64, 32, 8, 128, 8192), (1, 128, 1, 256, 1 << 30)])
def test_a_workspace_too_small_is_refused(lib, seqs, q_heads, heads, dim, tokens):
    need = ff.featfix_op_kv_attention_workspace(seqs, q_heads, heads, dim, tokens)
    assert 0 <= need < 1 << 30
    if need == 0:
        return
    c = dict(CACHE, seqs=seqs, heads=heads, head_dim=dim, table_pages=tokens // 16, ld_table=tokens // 16,
             k_stride=(1 << 20, 1 << 16, dim), v_stride=(1 << 20, 1 << 16, dim))
    good = dict(ATTN, cache=c, heads=q_heads, ldq=q_heads * dim, ldo=q_heads * dim, bytes=need)
    for bad in (dict(bytes=need - 1), dict(ws=NULL), dict(ws=P + 8)):
        assert call(lib, "featfix_op_kv_attention", {**good, **bad}) == ff.ERR_INVALID_ARG


def test_workspace_of_nothing(lib):
    for bad in ((0, 4, 4, 64, 100), (1, 5, 4, 64, 100), (1, 4, 0, 64, 100), (1, 4, 4, 512, 100), (1, 4, 4, 64, 0), (-1, 4, 4, 64, 9)):
        assert ff.featfix_op_kv_attention_workspace(*bad) == 0


def test_binding_refuses_wrong_tensors(lib):
    k8, sc = torch.zeros((4, 16, 2, 64), dtype=torch.uint8), torch.zeros((4, 16, 2))
    cache, table, lens = (k8, sc, k8, sc), torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    x, y = torch.zeros((3, 128)), torch.zeros((3, 256))
    bad = [lambda: ff.featfix_op_kv_write("f32", x, x, cache, table, lens),                          # not on a GPU
           lambda: ff.featfix_op_kv_write("f32", x, x, (k8, sc, k8), table, lens),
           lambda: ff.featfix_op_kv_write("f32", x, x, [k8, sc, k8, sc], table, lens),
           lambda: ff.featfix_op_kv_read("f32", (k8, sc, k8[:3], sc), table, lens, x, x),
           lambda: ff.featfix_op_kv_attention("f32", y, (k8, sc[..., 0], k8, sc), table, lens, y, None, 1.0),
           lambda: ff.featfix_op_kv_attention("f32", y, cache, table[0], lens, y, None, 1.0),
           lambda: ff.featfix_op_block_norms("f32", x, x[:2], 1e-6, out=x),
           lambda: ff.featfix_op_block_norms("bf16", x, x, 1e-6, out=x),
           lambda: ff.featfix_op_block_norms("f32", x, x, 1e-6, q=x)]
    for b in bad:
        with pytest.raises(ff.FeatFixError) as e:
            b()
        assert e.value.status == ff.ERR_INVALID_ARG
