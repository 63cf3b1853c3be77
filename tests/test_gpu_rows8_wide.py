"""The quantiser on rows wider than registers hold."""

import pytest
import torch

from paper_2607_27842_gb300 import featfix as ff

from .test_gpu_ops8 import TD, check8, held, held8, nb, randn, untouched

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,extra", [(1, 16385, 0), (3, 20001, 3), (2, 40000, 8), (5, 32768, 0), (2, 49153, 1)])
def test_quant8_wide_rows(cuda, dtype, rows, cols, extra):
    """More than one run of 16384 columns, whole blocks and a last one of a single column."""
    x = held(rows, cols, TD[dtype], extra)
    x.copy_(randn((rows, cols), 8) * torch.exp(randn((1, cols), 9, 2.0)))
    q, s = held8(rows, cols, 16), torch.empty((nb(cols), rows), device=cuda)
    ff.featfix_op_quant8(dtype, x, q, s)
    check8(q, s, x.double(), 1, x.double() * 0)
    assert untouched(q)
