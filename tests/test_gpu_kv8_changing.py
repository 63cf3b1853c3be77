"""Lengths that another stream changes while the 8-bit cache's operators run: the results of
those sequences mean nothing, but nothing outside of them is written, whether the attention
has a workspace or needs none, and later calls are as ever."""

import pytest
import torch

from paper_2607_27842_gb300 import featfix as ff

from .kv_helpers import Cache, NAN8, TD
from .test_gpu_kv8 import attend, randn, starts, work

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seqs,most,heads,group,dim,window,needs", [
    (1, 257, 4, 4, 128, 0, False),        # several warps to a unit, no workspace
    (5, 1500, 2, 3, 72, 100, True),       # whole units by the window alone
    (700, 60, 4, 1, 32, 0, False),        # more whole units than warps
    (3, 5000, 4, 4, 64, 0, True),         # shared out over all blocks
    (40, 2000, 8, 2, 128, 0, True)])
def test_lengths_that_change_during_calls(cuda, dtype, seqs, most, heads, group, dim, window, needs):
    g = torch.Generator().manual_seed(seqs)
    lens = [int(v) for v in torch.randint(1, most + 1, (seqs,), generator=g)]
    c = Cache(sum(-(-n // 16) for n in lens) + 1, 16, heads, dim, seqs, -(-most // 16))
    c.place(lens)
    c.fill(1)
    c.table[c.table == 1 << 30] = 0       # (a sequence may be longer for a while than its pages)
    width = heads * group * dim
    q = randn((seqs, width), 2).to(TD[dtype])
    want, _ = attend(c, q, heads * group, window=window)
    ws = work(c, heads * group)
    assert (ws.numel() > 0) == needs
    guarded = torch.full((seqs + 2, width + 16), 3.0, device="cuda").to(TD[dtype])
    out, bounds = guarded[1:-1, :width], torch.full((ws.numel() + 512,), 7, dtype=torch.uint8, device="cuda")
    ws = bounds[256:256 + ws.numel()] if needs else None
    states = [torch.tensor(s, dtype=torch.int32).cuda() for s in (
        [0] * seqs, lens, [1 << 30] * seqs, lens[::-1], [-5] * seqs, [most] * seqs, [n // 2 for n in lens])]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call = lambda: ff.featfix_op_kv_attention(dtype, q, c.parts, c.table, c.lens, out, ws, dim ** -0.5, window)
    for i in range(150):
        with torch.cuda.stream(side):
            for s in states:
                c.lens.copy_(s)
        for _ in range(4):
            call()
    torch.cuda.synchronize()
    assert (guarded[0] == 3).all() and (guarded[-1] == 3).all() and (guarded[:, width:] == 3).all()
    assert (bounds[:256] == 7).all() and (bounds[-256:] == 7).all()
    c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    call()
    assert (out == want).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ragged", [False, True])
def test_lengths_that_change_during_writes_and_reads(cuda, dtype, ragged):
    seqs, heads, dim, page = 60, 5, 72, 16
    counts = [(7 * b) % 23 for b in range(seqs)] if ragged else [1] * seqs
    lens = [n + 3 * b for b, n in enumerate(counts)]
    c = Cache(sum(-(-n // page) for n in lens) + 1, page, heads, dim, seqs, -(-max(lens) // page))
    c.place(lens)
    free = set(range(c.pages)) - {int(p) for b, n in enumerate(lens) for p in c.table[b, :-(-n // page)]}
    c.table[c.table == 1 << 30] = min(free)      # (for a while sequences are longer than their pages)
    k = randn((sum(counts), heads * dim), 3).to(TD[dtype])
    rs = starts(counts) if ragged else None
    back = torch.full((2, k.shape[0] + 2, k.shape[1] + 8), 3.0, device="cuda").to(TD[dtype])
    kb, vb = (t[1:-1, :k.shape[1]] for t in back)
    write = lambda: ff.featfix_op_kv_write(dtype, k, -k, c.parts, c.table, c.lens, row_start=rs)
    read = lambda: ff.featfix_op_kv_read(dtype, c.parts, c.table, c.lens, kb, vb, row_start=rs)
    states = [torch.tensor(s, dtype=torch.int32).cuda() for s in ([0] * seqs, lens, [1 << 30] * seqs, lens[::-1], [-5] * seqs)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for i in range(300):
        with torch.cuda.stream(side):
            for s in states:
                c.lens.copy_(s)
        for _ in range(3):
            write()
            read()
    torch.cuda.synchronize()
    assert (back[:, 0] == 3).all() and (back[:, -1] == 3).all() and (back[:, :, k.shape[1]:] == 3).all()
    base = c.k8._base
    while base._base is not None:
        base = base._base
    assert (base[..., dim:] == NAN8).all()
    c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    write()
    read()
    assert (kb == -vb).all() and ((kb - k).abs().amax(-1) <= k.abs().amax(-1) / 16).all()
