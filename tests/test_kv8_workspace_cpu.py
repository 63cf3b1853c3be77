"""How much scratch the attention over the 8-bit cache asks for (no GPU needed)."""

import pytest

from paper_2607_27842_gb300 import featfix as ff

from .test_kv8_cpu import ATTN, CACHE, P, call, lib  # noqa: F401  (lib: the fixture)

NEED = ff.featfix_op_kv_attention_workspace


@pytest.mark.parametrize("seqs,q_heads,heads,dim,tokens", [(1, 16, 4, 128, 131072), (64, 32, 8, 128, 8192), (1, 128, 1, 256, 1 << 30),
                                                           (1, 4, 4, 128, 1025), (4096, 32, 8, 128, 64)])
def test_long_caches_need_some_and_refuse_less(lib, seqs, q_heads, heads, dim, tokens):  # noqa: F811
    need = NEED(seqs, q_heads, heads, dim, tokens)
    assert 0 < need < 1 << 30
    c = dict(CACHE, seqs=seqs, heads=heads, head_dim=dim, page_size=1, table_pages=tokens, ld_table=tokens,
             k_stride=(1 << 20, 1 << 16, dim), v_stride=(1 << 20, 1 << 16, dim))
    good = dict(ATTN, cache=c, heads=q_heads, ldq=q_heads * dim, ldo=q_heads * dim, bytes=need)
    n0 = ff.featfix_launch_count()
    for bad in (dict(bytes=need - 1), dict(bytes=0), dict(ws=None), dict(ws=P + 8)):
        assert call(lib, "featfix_op_kv_attention", {**good, **bad}) == ff.ERR_INVALID_ARG
    assert ff.featfix_launch_count() == n0


@pytest.mark.parametrize("seqs,q_heads,heads,dim,tokens", [(1, 16, 4, 128, 257), (1, 16, 4, 128, 1024), (256, 32, 8, 128, 256),
                                                           (1, 1, 1, 256, 512), (4096, 8, 1, 64, 32)])
def test_short_caches_need_none(lib, seqs, q_heads, heads, dim, tokens):  # noqa: F811
    assert NEED(seqs, q_heads, heads, dim, tokens) == 0


@pytest.mark.parametrize("q_heads,heads,dim", [(16, 4, 128), (32, 8, 64), (9, 9, 40), (40, 2, 64), (128, 1, 256), (5, 1, 80)])
def test_more_sequences_or_tokens_never_need_less(lib, q_heads, heads, dim):  # noqa: F811
    """A workspace for up to `seqs` sequences of up to `tokens` tokens serves all smaller calls."""
    seqs = [1, 2, 3, 7, 16, 64, 151, 152, 153, 400, 1000, 4096, 30000]
    tokens = [1, 31, 32, 33, 64, 256, 500, 512, 513, 1000, 1024, 1025, 2000, 8192, 131072, 1 << 30]
    table = [[NEED(s, q_heads, heads, dim, t) for t in tokens] for s in seqs]
    for row in table:
        assert row == sorted(row) and row[-1] > 0
    for column in zip(*table):
        assert list(column) == sorted(column)


@pytest.mark.parametrize("bad", [(1, 4, 4, 12, 4096), (1, 4, 4, 264, 4096), (1, 70000, 4, 64, 4096), (1, 4, 3, 64, 4096),
                                 (1, 4, 4, 64, 1 << 31), (-1, 4, 4, 64, 4096), (1, 4, 4, 64, -5)])
def test_arguments_that_the_operator_refuses_need_none(lib, bad):  # noqa: F811
    assert NEED(*bad) == 0
