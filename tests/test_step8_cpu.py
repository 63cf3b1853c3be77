"""The 8-bit cache's book-keeping (step8.KVCache8), which needs no GPU."""

import pytest

from paper_2607_27842_gb300 import step8


def state(c):
    return list(c.free), [list(h) for h in c.held], list(c.used), c.table.tolist(), c.lens.tolist()


@pytest.mark.parametrize("counts", [[], [1], [1, 1, 1], [1, -1], [-1, 0], [1, 1.5], [1, None], [0, "1"]])
def test_counts_that_no_batch_has_are_refused(counts):
    c = step8.KVCache8(1, 6, 4, 1, 64, 2, 12, device="cpu")
    c.grow([3, 5])
    before = state(c)
    with pytest.raises(ValueError):
        c.grow(counts)
    assert state(c) == before
    c.grow([1, 0])
    assert c.used == [4, 5] and c.lens.tolist() == [4, 5]


def test_growing_and_dropping():
    c = step8.KVCache8(1, 6, 4, 1, 64, 3, 12, device="cpu")
    c.grow((4, 0, 9))
    assert c.lens.tolist() == [4, 0, 9]
    for b, n in enumerate((1, 0, 3)):
        assert c.table[b].tolist() == c.held[b] + [-1] * (3 - n) and len(c.held[b]) == n
    assert len(set(c.held[0] + c.held[2])) == 4
    c.drop(2)
    c.grow([1, 12, 0])
    assert c.lens.tolist() == [5, 12, 0] and c.table[2].tolist() == [-1] * 3
    assert c.table[:2].tolist() == [c.held[0] + [-1], c.held[1]] and not c.free[1:]
