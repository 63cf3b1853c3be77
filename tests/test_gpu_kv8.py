"""The 8-bit key-value cache through the C ABI: writing, reading and the attention
of one new token, each against its formula in float64.

What the calls may not read (places behind a sequence's end, padding of heads, table
places behind its end) holds NaN or numbers of no page in every test."""

import math

import pytest
import torch

from paper_2607_27842_gb300 import featfix as ff

from .kv_helpers import Cache, F8, NAN8, TD, U, attention, quant

pytestmark = pytest.mark.gpu


def randn(dims, seed, scale=1.0):
    return (torch.randn(dims, generator=torch.Generator().manual_seed(seed)) * scale).cuda()


def starts(counts, first=0):
    return torch.tensor([first + sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32).cuda()


def work(cache, q_heads):
    n = ff.featfix_op_kv_attention_workspace(cache.lens.numel(), q_heads, cache.heads, cache.dim,
                                             cache.table.shape[1] * cache.page)
    return torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")   # NaN in every type


def attend(cache, q, q_heads, scale=None, window=0, want_lse=True, dtype=None, out=None, **kw):
    dtype = dtype or ("f32" if q.dtype == torch.float32 else "bf16")
    out = torch.full_like(q, 3.0) if out is None else out
    lse = torch.full((q.shape[0], q_heads), 3.0, device="cuda") if want_lse else None
    scale = cache.dim ** -0.5 if scale is None else scale
    ff.featfix_op_kv_attention(dtype, q, cache.parts, cache.table, cache.lens, out, work(cache, q_heads), scale, window,
                               lse, **kw)
    return out, lse


def check_attention(cache, q, q_heads, scale=None, window=0):
    scale = cache.dim ** -0.5 if scale is None else scale
    dtype = "f32" if q.dtype == torch.float32 else "bf16"
    out, lse = attend(cache, q, q_heads, scale, window)
    want, want_lse, eo, el = attention(cache, q, q_heads, scale, window, dtype)
    assert ((out.double() - want).abs() <= eo).all(), float(((out.double() - want).abs() / (eo + 1e-300)).max())
    same = (lse.double() == want_lse) | ((lse.double() - want_lse).abs() <= el)
    assert same.all()
    return out, lse


# ----------------------------------------------------------------------------
# writing and reading
# ----------------------------------------------------------------------------

ROWS = [  # heads, dim, page, counts, lens behind the write
    (1, 8, 1, [1], [1]), (4, 128, 64, [1], [301]), (2, 64, 16, [1, 1, 1], [16, 17, 1]), (3, 72, 24, [5, 0, 40], [5, 3, 64]),
    (5, 80, 7, [13, 1, 0, 29], [20, 1, 0, 29]), (2, 256, 8, [9, 30], [17, 64]), (16, 96, 128, [200, 77], [333, 77]),
    (1, 16, 3, [4] * 65, list(range(4, 69))), (8, 200, 32, [33], [64])]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["token", "head", "gap"])
@pytest.mark.parametrize("heads,dim,page,counts,lens", ROWS)
def test_write_then_read(cuda, dtype, layout, heads, dim, page, counts, lens):
    c = Cache(sum(-(-n // page) for n in lens) + 2, page, heads, dim, len(lens), max(-(-n // page) for n in lens) + 1, layout)
    c.place(lens)
    rows, td = sum(counts), TD[dtype]
    spare = 3                                         # rows before the first sequence and behind the last
    qkv = torch.empty((rows + 2 * spare, 3 * heads * dim + 8), device="cuda").to(td)
    qkv.copy_(randn(qkv.shape, 3, 2.0) * torch.exp(randn((qkv.shape[0], 1), 4)))
    k, v = qkv[:, heads * dim:2 * heads * dim], qkv[:, 2 * heads * dim:3 * heads * dim]
    row_start = starts(counts, spare)
    ff.featfix_op_kv_write(dtype, k, v, c.parts, c.table, c.lens, row_start=row_start)
    seen = torch.zeros((c.pages, page), dtype=torch.bool, device="cuda")
    at = spare
    for b, (n, total) in enumerate(zip(counts, lens)):
        place = c.at(b, total - n, total)
        seen[place] = True
        for x, q8, scale in ((k, c.k8, c.k_scale), (v, c.v8, c.v_scale)):
            x = x[at:at + n].reshape(n, heads, dim)
            _, want = quant(x)
            # the scale: one rounded product; a value: half a step of it
            assert ((scale[place].double() / want.double() - 1).abs() <= 2.0 ** -22).all()
            got = q8[place].view(F8).double() * scale[place].double()[..., None]
            tol = torch.maximum(x.double().abs() * 2.0 ** -4, want.double()[..., None] * 2.0 ** -10) * 1.001
            assert ((got - x.double()).abs() <= tol).all()
        at += n
    # nothing else was written
    for q8, scale in ((c.k8, c.k_scale), (c.v8, c.v_scale)):
        assert (q8[~seen] == NAN8).all() and scale[~seen].isnan().all()
        base = q8._base
        while base._base is not None:
            base = base._base
        assert (base[..., dim:] == NAN8).all()

    back = torch.full((rows + 2 * spare, 2 * heads * dim + 8), 3.0, device="cuda").to(td)
    kb, vb = back[:, :heads * dim], back[:, heads * dim:2 * heads * dim]
    ff.featfix_op_kv_read(dtype, c.parts, c.table, c.lens, kb, vb, row_start=row_start)
    at = spare
    for b, (n, total) in enumerate(zip(counts, lens)):
        for x, want in zip((kb, vb), c.values(b, total - n, total)):
            got = x[at:at + n].double().view(n, heads, dim)
            assert ((got - want).abs() <= want.abs() * (U[dtype] + 2.0 ** -24) * 1.001).all()
        at += n
    assert (back[:spare] == 3).all() and (back[at:] == 3).all() and (back[:, 2 * heads * dim:] == 3).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_off_vector_boundaries(cuda, dtype):
    """Row strides and starts of single elements."""
    c = Cache(9, 16, 3, 72, 2, 4)
    c.place([40, 50])
    base = randn((70, 2 * 216 + 3), 5).to(TD[dtype])
    k, v = base[:, 1:217], base[:, 218:434]
    rs = starts([30, 40])
    ff.featfix_op_kv_write(dtype, k, v, c.parts, c.table, c.lens, row_start=rs)
    other = Cache(9, 16, 3, 72, 2, 4)
    other.place([40, 50])
    ff.featfix_op_kv_write(dtype, k.contiguous(), v.contiguous(), other.parts, other.table, other.lens, row_start=rs)
    assert (c.k8 == other.k8).all() and (c.v8 == other.v8).all()
    a = torch.full_like(base, 3.0)
    b = torch.full((70, 432), 3.0, device="cuda").to(TD[dtype])
    ff.featfix_op_kv_read(dtype, c.parts, c.table, c.lens, a[:, 1:217], a[:, 218:434], row_start=rs)
    ff.featfix_op_kv_read(dtype, c.parts, c.table, c.lens, b[:, :216], b[:, 216:], row_start=rs)
    assert (a[:, 1:217] == b[:, :216]).all() and (a[:, 218:434] == b[:, 216:]).all()
    assert (a[:, 0] == 3).all() and (a[:, 217] == 3).all() and (a[:, 434] == 3).all()


def test_special_values_and_places_that_are_not_there(cuda):
    """NaN and infinities make all of their head NaN; zeros and denormals keep the least scale; tokens
    before the first, in no page and past the table's end are skipped, and read as zeros."""
    c = Cache(4, 4, 2, 16, 4, 2)
    c.place([4, 2, 8, 0])
    c.lens[2] = 11                                    # the table holds 8
    c.table[0, 0] = -1                                # no page
    counts = [4, 5, 5, 2]                             # sequence 1 has 2 tokens, sequence 3 none
    k = randn((16, 32), 6)
    k[4 + 3, :16] = 0
    k[4 + 3, 3] = math.nan
    k[4 + 4, :16] = 0
    k[4 + 4, 16] = -math.inf
    v = torch.zeros_like(k)
    v[9 + 4, 5] = 1e-38
    ff.featfix_op_kv_write("f32", k, v, c.parts, c.table, c.lens, row_start=starts(counts))
    p, s = c.at(1, 0, 2)
    assert c.k_scale[p, s][0, 0].isnan() and c.k_scale[p, s][1, 1].isinf() and c.k_scale[p, s][1, 0] == 2.0 ** -100
    back = [torch.full((16, 32), 3.0, device="cuda") for _ in range(2)]
    ff.featfix_op_kv_read("f32", c.parts, c.table, c.lens, *back, row_start=starts(counts))
    kb, vb = back
    assert (kb[:4] == 0).all() and (kb[4:7] == 0).all() and (kb[14:] == 0).all()
    assert kb[7, :16].isnan().all() and not kb[7, 16:].isnan().any()
    assert (kb[8, :16] == 0).all() and kb[8, 16:].isnan().all()
    # lengths past the table count to its end: rows 9 .. 13 are tokens 3 .. 7
    want, sc = quant(k[9:14].view(5, 2, 16))
    assert ((kb[9:14].view(5, 2, 16) - want.float() * sc[..., None]).abs() <= sc[..., None] * 32).all()
    assert (vb == 0).all() or ((vb - v).abs() <= 2.0 ** -100).all()
    out, lse = attend(c, randn((4, 32), 7), 2, window=5)   # (of sequence 2 only what was written)
    assert (out[0] == 0).all() and (lse[0] == -math.inf).all()
    assert out[1].isnan().all() and lse[1].isnan().all()
    assert out[2].isfinite().all() and (out[3] == 0).all() and (lse[3] == -math.inf).all()


# ----------------------------------------------------------------------------
# attention
# ----------------------------------------------------------------------------

ATTENTION = [  # q heads, heads, dim, page, lens, window
    (1, 1, 8, 1, [1], 0), (4, 4, 128, 64, [1, 2, 0, 63, 64, 65], 0), (16, 4, 128, 64, [257], 0), (16, 4, 128, 16, [3000], 0),
    (32, 8, 128, 16, [513, 0, 1, 1024, 77, 2000, 15], 0), (6, 2, 72, 24, [100, 700, 33], 0), (5, 1, 80, 7, [333, 128, 129], 50),
    (16, 1, 256, 32, [1, 500, 31], 0), (40, 2, 64, 128, [127, 128, 999], 0), (3, 3, 96, 8, [40] * 9, 17),
    (8, 1, 200, 1, [130, 5], 1), (17, 1, 32, 16, [1000, 6], 0), (2, 2, 16, 3, [10, 300], 1000), (34, 2, 136, 5, [88, 1], 31),
    (16, 16, 72, 32, [700, 256, 300], 256), (1, 1, 128, 64, [9000], 0), (128, 1, 64, 64, [450, 20], 0), (9, 9, 40, 16, [350] * 33, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q_heads,heads,dim,page,lens,window", ATTENTION)
def test_attention(cuda, dtype, q_heads, heads, dim, page, lens, window):
    for i, layout in enumerate(("token", "head", "gap")):
        c = Cache(sum(-(-n // page) for n in lens) + 2, page, heads, dim, len(lens), max(-(-n // page) for n in lens) + i, layout)
        c.place(lens, i)
        c.fill(i)
        q = randn((len(lens), q_heads * dim + 24), 8 + i, 1.5).to(TD[dtype])[:, 8:8 + q_heads * dim]
        check_attention(c, q, q_heads, window=window)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,seqs,heads,group", [(20000, 1, 2, 4), (20000, 3, 1, 1), (70000, 1, 1, 8)])
def test_long_caches(cuda, dtype, tokens, seqs, heads, group):
    """One sequence shared out over many blocks."""
    lens = [tokens - 777 * i for i in range(seqs)]
    c = Cache(sum(-(-n // 64) for n in lens), 64, heads, 128, seqs, -(-tokens // 64))
    c.place(lens)
    c.fill(2)
    q = randn((seqs, heads * group * 128), 9, 2.0).to(TD[dtype])
    check_attention(c, q, heads * group)
    # the table's width alone decides how the work is shared out: short rows in a wide table
    c.lens.copy_(torch.tensor([5] + [0] * (seqs - 1)))
    check_attention(c, q, heads * group)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_missing_pages_and_nan_are_masked_or_seen(cuda, dtype):
    """Tokens of no page are masked, a whole row of them too; NaN and infinite scales of visible
    tokens make the row NaN, behind the window they do nothing."""
    c = Cache(40, 16, 2, 64, 4, 12)
    c.place([150, 100, 100, 64])
    c.fill(3)
    c.table[0, 3] = -1
    c.table[0, 8] = 40
    c.table[3, :4] = torch.tensor([-5, 1 << 30, 41, -(1 << 31)], dtype=torch.int32)
    c.k_scale[c.at(1, 20, 21)] = math.nan
    c.v_scale[c.at(2, 20, 21)] = math.inf
    q = randn((4, 8 * 64), 10, 1.5).to(TD[dtype])
    out, lse = attend(c, q, 8)
    want, want_lse, eo, el = attention(c, q, 8, 0.125, 0, dtype)
    for b in (0, 3):
        assert ((out[b].double() - want[b]).abs() <= eo[b]).all()
        assert ((lse[b].double() == want_lse[b]) | ((lse[b].double() - want_lse[b]).abs() <= el[b])).all()
    assert (out[3] == 0).all()
    assert out[1].isnan().all() and out[2].isnan().all()
    seen, _ = attend(c, q, 8, window=79)
    assert seen.isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q_size,k_size,v_size,scale", [(1e18, 1e-18, 1.0, 0.1), (1e-30, 1e30, 1e25, 0.1), (1.0, 1.0, 1e-30, 0.1),
                                                        (1e-3, 1e-3, 1.0, 1.0), (30.0, 1.0, 1.0, 0.125), (1.0, 1.0, 1.0, -0.1),
                                                        (1.0, 1.0, 1.0, 0.0)])
def test_magnitudes(cuda, dtype, q_size, k_size, v_size, scale):
    c = Cache(30, 16, 2, 64, 2, 14)
    c.place([200, 201])
    c.fill(4, 1.0)
    c.k_scale.mul_(k_size)
    c.v_scale.mul_(v_size)
    check_attention(c, randn((2, 8 * 64), 11, q_size).to(TD[dtype]), 8, scale=scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_of_very_different_size(cuda, dtype):
    """A token with most of the probability and values near zero beside tokens of large values, and
    values 2^60 apart."""
    c = Cache(30, 16, 1, 64, 2, 14)
    c.place([200, 201])
    c.fill(5)
    q = randn((2, 4 * 64), 12, 1.5).to(TD[dtype])
    k0 = q.float().view(2, 4, 64)[:, 0]
    for b in range(2):
        page, slot = c.at(b, 0, 1)
        q8, s = quant(k0[b])
        c.k8[page, slot, 0] = q8.view(torch.uint8)
        c.k_scale[page, slot, 0] = s * 4
        c.v_scale[page, slot, 0] *= 1e-4
        c.v_scale[c.at(b, 50, 100)] *= 2.0 ** (-60 * b)
    check_attention(c, q, 4)


def test_offsets_past_32_bits(cuda):
    """Pages 3 GB apart: places lie past 2^32 bytes, scales past 2^31 elements of their buffer."""
    heads, dim, page = 1, 64, 16
    kv = torch.zeros(3 * (3 << 30) + (1 << 20), dtype=torch.uint8, device="cuda")
    sc = torch.zeros(3 * (3 << 28) + (1 << 16), dtype=torch.float32, device="cuda")
    c = Cache(4, page, heads, dim, 1, 4)
    c.place([60])
    pools = []
    for i, (q8, s) in enumerate(((c.k8, c.k_scale), (c.v8, c.v_scale))):
        q = torch.as_strided(kv, (4, page, heads, dim), (3 << 30, dim, dim, 1), i * (page * dim))
        z = torch.as_strided(sc, (4, page, heads), (3 << 28, heads, heads), i * page)
        pools += [q, z]
    c.k8, c.k_scale, c.v8, c.v_scale = pools
    k, v = randn((60, 64), 13).bfloat16(), randn((60, 64), 14).bfloat16()
    ff.featfix_op_kv_write("bf16", k, v, c.parts, c.table, c.lens, row_start=starts([60]))
    kb, vb = torch.empty_like(k), torch.empty_like(v)
    ff.featfix_op_kv_read("bf16", c.parts, c.table, c.lens, kb, vb, row_start=starts([60]))
    for a, b in ((k, kb), (v, vb)):
        assert ((a - b).double().abs() <= a.double().abs() * (2.0 ** -4 + 2.0 ** -7) + 0.02 * 2.0 ** -10).all()
    check_attention(c, randn((1, 4 * 64), 15).bfloat16(), 4)


def test_in_place_other_streams_and_no_lse(cuda):
    c = Cache(40, 16, 4, 128, 3, 12)
    c.place([190, 1, 77])
    c.fill(6)
    q = randn((3, 16 * 128), 16).bfloat16()
    want, _ = attend(c, q, 16)
    x = q.clone()
    attend(c, x, 16, out=x, want_lse=False)
    assert (x == want).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y, _ = attend(c, q, 16)
    z = torch.empty_like(q)
    ff.featfix_op_kv_attention("bf16", q, c.parts, c.table, c.lens, z, work(c, 16), 128 ** -0.5, stream=side)
    torch.cuda.synchronize()
    assert (y == want).all() and (z == want).all()


def test_no_sequences(cuda):
    c = Cache(2, 16, 4, 128, 1, 2)
    none = torch.empty((0, 2), dtype=torch.int32, device="cuda")
    lens = torch.empty((0,), dtype=torch.int32, device="cuda")
    q = torch.empty((0, 512), device="cuda")
    n0 = ff.featfix_launch_count()
    ff.featfix_op_kv_attention("f32", q, c.parts, none, lens, q, None, 1.0)
    ff.featfix_op_kv_write("f32", q, q, c.parts, none, lens)
    ff.featfix_op_kv_read("f32", c.parts, none, lens, q, q)
    assert ff.featfix_launch_count() == n0


@pytest.mark.parametrize("seqs,table_pages", [(2, 40), (1, 600)])
def test_a_captured_step_follows_table_and_lengths(cuda, seqs, table_pages):
    """Write and attention captured once, then replayed while sequences grow into new pages; every
    replay equals the eager call bit for bit, and a padded place (length 0) gives zeros."""
    c = Cache(seqs * table_pages, 16, 2, 64, seqs, table_pages)
    c.place([16 * table_pages] * seqs)
    k, v, q = (randn((seqs, n * 64), 17 + n).bfloat16() for n in (2, 2, 8))
    out, lse, ws = torch.empty_like(q), torch.empty((seqs, 8), device="cuda"), work(c, 8)

    def step(o):
        ff.featfix_op_kv_write("bf16", k, v, c.parts, c.table, c.lens)
        ff.featfix_op_kv_attention("bf16", q, c.parts, c.table, c.lens, o, ws, 0.125, lse=lse)

    c.lens.fill_(1)
    step(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out)
    for n in range(1, 40):
        c.lens.fill_(n)
        if seqs > 1 and n == 20:
            c.lens[1] = 0
        for t, s in ((k, 1), (v, 2), (q, 3)):
            t.copy_(randn(t.shape, 100 * n + s))
        graph.replay()
        eager = torch.empty_like(q)
        got = out.clone()
        step(eager)
        assert (eager == got).all()
        if n == 20 and seqs > 1:
            assert (got[1] == 0).all()
            c.lens.fill_(n)
            ff.featfix_op_kv_write("bf16", k, v, c.parts, c.table, c.lens)
        if n in (1, 2, 16, 17, 39):
            check_attention(c, q, 8)


def test_same_inputs_give_the_same_bits(cuda):
    lens = [5000, 1, 300, 0, 2222, 64]
    c = Cache(sum(-(-n // 16) for n in lens), 16, 8, 128, 6, 313)
    c.place(lens)
    c.fill(7)
    q = randn((6, 32 * 128), 18, 1.5).bfloat16()
    first, lse = attend(c, q, 32)
    for _ in range(20):
        again, l2 = attend(c, q, 32)
        assert (again == first).all() and (l2 == lse).all()
