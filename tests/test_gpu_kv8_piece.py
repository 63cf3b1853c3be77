"""Several new tokens of one sequence at a time: written as rows of the sequence, and
attended as sequences of their own over the same pages."""

import pytest
import torch

from paper_2607_27842_gb300 import featfix as ff

from .kv_helpers import Cache, TD
from .test_gpu_kv8 import check_attention, randn, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("had,new,heads,group,dim,page", [(0, 1, 2, 2, 64, 16), (100, 40, 4, 4, 128, 16), (0, 300, 2, 8, 72, 24),
                                                         (5000, 70, 2, 4, 128, 64)])
def test_a_piece(cuda, dtype, had, new, heads, group, dim, page):
    one = Cache(-(-(had + new) // page), page, heads, dim, 1, -(-(had + new) // page))
    one.place([had + new])
    if had:
        one.fill(4)
    k, v = (randn((new, heads * dim), 30 + i).to(TD[dtype]) for i in range(2))
    ff.featfix_op_kv_write(dtype, k, v, one.parts, one.table, one.lens, row_start=starts([new]))
    q = randn((new, heads * group * dim), 33, 1.5).to(TD[dtype])
    piece = Cache(1, page, heads, dim, new, one.table.shape[1])
    piece.k8, piece.k_scale, piece.v8, piece.v_scale, piece.pages = *one.parts, one.pages
    piece.table = one.table.repeat(new, 1)
    piece.lens = torch.arange(had + 1, had + new + 1, dtype=torch.int32, device="cuda")
    check_attention(piece, q, heads * group)
    check_attention(one, q[-1:], heads * group)      # as the sequence's only new token
