"""The key-value cache's operators and the block norms as programs call them: many
sequences, several threads and streams, tensors of another GPU, queries that are no numbers."""

import math
import threading

import pytest
import torch

from paper_2607_27842_gb300 import featfix as ff

from .kv_helpers import Cache, F8, TD, attention
from .test_gpu_kv8 import attend, check_attention, randn, starts, work
from .test_gpu_ops8_device import Elsewhere

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seqs,most,heads,group,dim,page,window", [
    (70, 1500, 2, 3, 64, 16, 0),        # shared out over all blocks, several sequences to a lane of the line
    (300, 90, 8, 1, 32, 8, 0),          # whole units, more than the SMs have warps
    (200, 2000, 1, 4, 128, 32, 70),     # short by the window alone
    (1100, 40, 2, 2, 128, 16, 0),
    (1200, 90, 8, 1, 32, 8, 0),         # shared out: more steps than whole units are taken for
    (900, 70, 9, 2, 64, 16, 40), (500, 120, 5, 9, 72, 8, 0)])
def test_many_sequences(cuda, dtype, seqs, most, heads, group, dim, page, window):
    g = torch.Generator().manual_seed(seqs)
    lens = [int(v) for v in torch.randint(0, most + 1, (seqs,), generator=g)]
    lens[3], lens[seqs // 2] = 0, most
    c = Cache(sum(-(-n // page) for n in lens) + 1, page, heads, dim, seqs, -(-most // page), "token")
    c.place(lens)
    c.fill(2)
    q = randn((seqs, heads * group * dim), 19, 1.5).to(TD[dtype])
    check_attention(c, q, heads * group, window=window)


@pytest.mark.parametrize("seqs", [1, 31, 32, 1023, 1024, 2500])
def test_rows_of_many_sequences(cuda, seqs):
    """The search for a row's sequence, empty ones among them, at the edges of its steps."""
    g = torch.Generator().manual_seed(seqs)
    counts = [int(v) for v in torch.randint(0, 3, (seqs,), generator=g)]
    counts[0] = 2
    lens = [n + i % 3 for i, n in enumerate(counts)]
    c = Cache(sum(-(-n // 2) for n in lens), 2, 1, 16, seqs, 2)
    c.place(lens)
    rows = sum(counts)
    k = randn((rows, 16), 20)
    ff.featfix_op_kv_write("f32", k, -k, c.parts, c.table, c.lens, row_start=starts(counts))
    kb, vb = torch.empty_like(k), torch.empty_like(k)
    ff.featfix_op_kv_read("f32", c.parts, c.table, c.lens, kb, vb, row_start=starts(counts))
    assert ((kb - k).abs() <= k.abs() * 2.0 ** -4 + 1e-4).all() and (vb == -kb).all()
    at = 0
    for b, (n, total) in enumerate(zip(counts, lens)):
        if n:
            assert (c.values(b, total - n, total)[0].float().view(n, 16) == kb[at:at + n]).all()
        at += n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_queries_that_are_no_numbers(cuda, dtype):
    """A NaN or an infinity makes its own query head NaN, no other."""
    c = Cache(30, 16, 2, 64, 3, 9)
    c.place([130, 140, 17])
    c.fill(8)
    q = randn((3, 8 * 64), 21).to(TD[dtype])
    want, _ = attend(c, q, 8)
    q[0, 5], q[1, 3 * 64 + 1], q[2] = math.nan, math.inf, 0
    out, lse = attend(c, q, 8)
    assert out[0, :64].isnan().all() and out[1, 3 * 64:4 * 64].isnan().all()
    assert (out[0, 64:] == want[0, 64:]).all() and (out[1, :3 * 64] == want[1, :3 * 64]).all()
    ref, ref_lse, eo, el = attention(c, q, 8, 0.125, 0, dtype)
    assert ((out[2].double() - ref[2]).abs() <= eo[2]).all() and ((lse[2].double() - ref_lse[2]).abs() <= el[2]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [-1.0, -math.inf, -1e-38, math.nan])
def test_scales_that_no_token_has(cuda, dtype, scale):
    """Negative scales are NaN, as infinite ones: in the head that has one, and in no other."""
    c = Cache(30, 16, 2, 64, 3, 9)
    c.place([130, 140, 17])
    c.fill(11)
    q = randn((3, 8 * 64), 22).to(TD[dtype])
    want, _ = attend(c, q, 8)
    (p, s), (p2, s2) = c.at(0, 77, 78), c.at(2, 16, 17)
    c.k_scale[p, s, 1] = scale
    c.v_scale[p2, s2, 0] = scale
    out, _ = attend(c, q, 8)
    assert out[0, 4 * 64:].isnan().all() and out[2, :4 * 64].isnan().all()
    assert (out[0, :4 * 64] == want[0, :4 * 64]).all() and (out[1] == want[1]).all() and (out[2, 4 * 64:] == want[2, 4 * 64:]).all()
    k, v = (torch.zeros((3, 128), device="cuda", dtype=TD[dtype]) for _ in range(2))
    ff.featfix_op_kv_read(dtype, c.parts, c.table, c.lens, k, v)
    assert not k.isnan().any() and v[2, :64].isnan().all() and not v[2, 64:].isnan().any() and not v[:2].isnan().any()


def test_streams_and_threads_with_workspaces_of_their_own(cuda):
    """Two threads, each on a stream with its own workspace and cache, at the same time."""
    caches, qs, wants = [], [], []
    for i in range(2):
        c = Cache(400, 16, 4, 128, 3, 140, "head" if i else "token")
        c.place([2200 - 300 * i, 77, 1500])
        c.fill(9 + i)
        caches.append(c)
        qs.append(randn((3, 16 * 128), 22 + i, 1.5).bfloat16())
        wants.append(attend(c, qs[i], 16)[0])
    torch.cuda.synchronize()
    streams, bad = [torch.cuda.Stream() for _ in range(2)], []
    start = threading.Barrier(2)

    def run(i):
        c, ws, out = caches[i], work(caches[i], 16), torch.empty_like(qs[i])
        x, s = qs[i].clone(), torch.empty_like(qs[i])
        with torch.cuda.stream(streams[i]):
            streams[i].wait_stream(torch.cuda.default_stream())
            start.wait()
            for k in range(300):
                ff.featfix_op_kv_attention("bf16", qs[i], c.parts, c.table, c.lens, out, ws, 128 ** -0.5)
                ff.featfix_op_block_norms("bf16", out, x, 1e-6, sum_out=s)
                if k % 50 == 0 and not bool((out == wants[i]).all()):
                    bad.append((i, k))

    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not bad


def test_tensors_of_another_gpu_are_refused(cuda):
    f32, bf16, u8, i32 = torch.float32, torch.bfloat16, torch.uint8, torch.int32
    sizes = {"x": ((3, 128), bf16), "q": ((3, 256), bf16), "k8": ((4, 16, 2, 64), u8), "s": ((4, 16, 2), f32), "table": ((3, 2), i32),
             "lens": ((3,), i32), "lse": ((3, 4), f32), "mod": ((1, 128), f32), "w": ((128,), bf16), "start": ((4,), i32)}
    near = {n: torch.zeros(d, dtype=t, device=cuda) for n, (d, t) in sizes.items()}
    far = {n: Elsewhere.of(d, t, "cuda:%d" % (torch.cuda.current_device() + 1)) for n, (d, t) in sizes.items()}
    cache = lambda t: (t["k8"], t["s"], near["k8"], near["s"])
    calls = {
        ("x", "k8", "s", "table", "lens", "start"): lambda t: ff.featfix_op_kv_write("bf16", t["x"], near["x"], cache(t), t["table"], t["lens"],
                                                                                     row_start=t["start"]),
        ("k8", "s", "table"): lambda t: ff.featfix_op_kv_read("bf16", cache(t), t["table"], t["lens"], near["x"], near["x"]),
        ("q", "lse", "lens", "w"): lambda t: ff.featfix_op_kv_attention("bf16", t["q"], cache(t), t["table"], t["lens"], near["q"], t["w"],
                                                                        1.0, lse=t["lse"]),
        ("x", "mod", "w"): lambda t: ff.featfix_op_block_norms("bf16", near["x"], t["x"], 1e-6, gate=t["mod"], weight=t["w"],
                                                               rows_per_batch=3, out=near["x"])}
    n0 = ff.featfix_launch_count()
    for names, call in calls.items():
        for name in names:
            with pytest.raises(ff.FeatFixError) as e:
                call({**near, name: far[name]})
            assert e.value.status == ff.ERR_INVALID_ARG and "GPU" in str(e.value), (name, str(e.value))
    assert ff.featfix_launch_count() == n0


def test_a_padded_batch_and_rows_of_no_sequence(cuda):
    """A batch of a fixed size whose last places are free: lengths of 0 and rows behind the last start.
    Nothing of theirs is written to the cache; their attention is zero; rows read are left alone."""
    c = Cache(12, 16, 2, 64, 5, 3)
    c.place([40, 3, 17, 0, 0])
    c.fill(11)
    before = [t.clone() for t in c.parts]
    k = randn((9, 128), 23).bfloat16()
    rs = torch.tensor([0, 2, 2, 5, 5, 5], dtype=torch.int32).cuda()      # rows 5 .. 8 are of no sequence
    ff.featfix_op_kv_write("bf16", k, k, c.parts, c.table, c.lens, row_start=rs)
    changed = (c.k8 != before[0]).any(-1).any(-1)
    allowed = torch.zeros_like(changed)
    for b, first, end in ((0, 38, 40), (2, 14, 17)):
        allowed[c.at(b, first, end)] = True
    assert not (changed & ~allowed).any()
    out = [torch.full((9, 128), 3.0, device="cuda").bfloat16() for _ in range(2)]
    ff.featfix_op_kv_read("bf16", c.parts, c.table, c.lens, *out, row_start=rs)
    assert all((t[5:] == 3).all() for t in out) and not any((t[:5] == 3).all(-1).any() for t in out)
    q = randn((5, 4 * 64), 24).bfloat16()
    o, lse = attend(c, q, 4)
    assert (o[3:] == 0).all() and (lse[3:] == -math.inf).all() and (o[:3] != 0).any(-1).all()
