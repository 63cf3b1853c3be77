"""Columns of a head that no axis turns: copied bit for bit, whatever they hold, and
without any effect on the columns that are turned."""

import math

import pytest
import torch

from paper_2607_27842_gb300 import featfix as ff

from .test_gpu_ops8 import TD, randn

pytestmark = pytest.mark.gpu

SPECIAL = [math.inf, -math.inf, math.nan, -0.0, 0.0, 1e-40, -3e38]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("hd,axes,extra", [(128, (54, 20), 0), (128, (64,), 0), (72, (10, 20, 16), 0), (256, (200, 54), 0),
                                           (34, (6, 12), 1), (40, (14, 8), 0), (128, (2,), 0), (80, (70,), 0)])
def test_columns_past_the_axes_are_copied(cuda, dtype, halves, hd, axes, extra):
    rows, heads, rot = 37, 5, sum(axes)
    x = randn((rows, heads * hd + extra), 3).to(TD[dtype])[:, :heads * hd]
    pos = torch.randint(0, 900, (len(axes), rows), generator=torch.Generator().manual_seed(4), dtype=torch.int32).cuda()

    def rope(v):
        o = torch.empty_like(v)
        ff.featfix_op_rope(dtype, pos, axes, hd, q=v, q_out=o, halves=halves)
        return o.reshape(rows, heads, hd)

    plain = rope(x)
    y = x.clone()
    tail = y.view(rows, heads, hd)[..., rot:]
    tail.copy_(torch.tensor(SPECIAL, device=cuda).to(TD[dtype])[
        torch.randint(0, len(SPECIAL), tail.shape, generator=torch.Generator().manual_seed(5)).cuda()])
    got = rope(y)
    assert torch.equal(got[..., :rot], plain[..., :rot])
    nan = torch.isnan(tail)
    assert torch.equal(torch.isnan(got[..., rot:]), nan)
    bits = torch.int32 if dtype == "f32" else torch.int16
    assert torch.equal(got[..., rot:].contiguous().view(bits)[~nan], tail.contiguous().view(bits)[~nan])
