"""What a step over the 8-bit cache leaves alone, and what its growth waits for."""

import pytest
import torch

from paper_2607_27842_gb300 import featfix as ff
from paper_2607_27842_gb300 import step8

from .test_gpu_step8 import weights

pytestmark = pytest.mark.gpu

C, M, HEADS, K_HEADS, DIM, PAGE, STEPS, SEQS = 256, 512, 4, 2, 64, 4, 12, 3


def model(seed=5):
    layers = [weights(C, M, HEADS, K_HEADS, DIM, seed + i) for i in range(2)]
    cache = step8.KVCache8(2, SEQS * 8, PAGE, K_HEADS, DIM, SEQS, 4 * STEPS)
    return step8.Step8(layers, HEADS, K_HEADS, cache), cache


def tokens():
    return torch.randn((STEPS, SEQS, C), generator=torch.Generator().manual_seed(6)).bfloat16().cuda()


@pytest.mark.parametrize("captured", [False, True])
def test_a_sequence_without_a_new_token_keeps_its_cache(cuda, captured):
    """Sequence 1 takes part in every other step only: the tokens it gets are those it gets where it always
    takes part, whatever its row holds in between."""
    x, (net, cache) = tokens(), model()
    want = []
    for i in range(STEPS):
        cache.grow([1] * SEQS)
        want.append(net(x[i].clone()))
    net, cache = model()
    buf, graph = x[0].clone(), None
    if captured:
        cache.grow([1, 1, 1])
        net(buf)                  # (modules loaded; the same token again below)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            net(buf)
    at = [0] * SEQS
    for i in range(2 * STEPS):
        on = [int(not (b == 1 and i % 2)) * int(at[b] < STEPS) for b in range(SEQS)]
        if not captured or i:
            cache.grow(on)
        for b in range(SEQS):
            buf[b] = x[at[b], b] if on[b] else 1e4
        kept = [(cache.k8[:, cache.held[b][-1]].clone(), cache.v_scale[:, cache.held[b][-1]].clone()) for b in range(SEQS)]
        graph.replay() if captured else net(buf)
        for b in range(SEQS):
            if on[b]:
                assert (buf[b] == want[at[b]][b]).all(), (i, b)
                at[b] += 1
            else:
                assert (cache.k8[:, cache.held[b][-1]] == kept[b][0]).all() and (cache.v_scale[:, cache.held[b][-1]] == kept[b][1]).all()
    assert at == [STEPS] * SEQS


def test_growing_twice_and_stepping_twice(cuda):
    """A step serves all that grew since the one before; run again it gives the same."""
    x, (net, cache) = tokens(), model()
    cache.grow([1, 1, 1])
    want = net(x[0].clone())
    net2, cache2 = model()
    cache2.grow([1, 0, 0])
    cache2.grow([0, 1, 0])
    cache2.grow([0, 0, 1])
    for _ in range(2):
        assert (net2(x[0].clone()) == want).all()
    cache.grow([1, 1, 1])
    cache2.grow([1, 1, 1])
    assert (net(x[1].clone()) == net2(x[1].clone())).all()
    cache.drop(1)
    cache.grow([1, 1, 1])         # another sequence in its place
    cache2.grow([1, 0, 1])
    a, b = net(x[2].clone()), net2(x[2].clone())
    assert (a[0] == b[0]).all() and (a[2] == b[2]).all()


def test_lengths_set_without_growing(cuda):
    """A program that keeps pages in hand and counts on the device writes every length's last token."""
    x, (net, cache) = tokens(), model()
    other, grown = model()
    cache.grow([STEPS] * SEQS)
    cache.lens.zero_()
    for i in range(4):
        cache.lens.add_(1)
        grown.grow([1] * SEQS)
        assert (net(x[i].clone()) == other(x[i].clone())).all()


def test_tokens_that_the_program_wrote_itself(cuda):
    """A prompt written with the operator's own call is no step's new token."""
    x, (net, cache) = tokens(), model()
    cache.grow([5, 0, 2])
    start = torch.tensor([0, 5, 5, 7], dtype=torch.int32, device="cuda")
    k = torch.randn((7, K_HEADS * DIM), generator=torch.Generator().manual_seed(8)).bfloat16().cuda()
    for i in range(2):
        ff.featfix_op_kv_write("bf16", k, -k, cache.layer(i), cache.table, cache.lens, row_start=start)
    cache.written()
    kept = [t.clone() for t in cache.layer(0)]
    net(x[0].clone())
    assert all((a == b).all() for a, b in zip(kept, cache.layer(0)))
    cache.grow([0, 1, 1])
    net(x[1].clone())
    mine = torch.tensor(cache.held[0], device="cuda")
    assert all((a[mine] == b[mine]).all() for a, b in zip(kept, cache.layer(0)))
    changed = (cache.layer(0)[0] != kept[0]).flatten(2).any(-1)
    where = {(cache.held[1][0], 0), (cache.held[2][0], 2)}
    assert {tuple(p) for p in changed.nonzero().tolist()} == where


def test_growing_waits_for_nothing(cuda):
    _, cache = model()
    cache.grow([1, 2, 3])         # (pinned memory is there from now on)
    cache.drop(0)
    torch.cuda.synchronize()
    mode = torch.cuda.get_sync_debug_mode()
    torch.cuda.set_sync_debug_mode("error")
    try:
        for i in range(20):
            cache.grow([1, int(i < 9), 0])
            if i == 9:
                cache.drop(1)
    finally:
        torch.cuda.set_sync_debug_mode(mode)
    assert cache.lens.tolist() == [20, 0, 3] and cache.table[0].tolist() == cache.held[0] + [-1] * (cache.width - 5)
