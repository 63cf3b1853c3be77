"""Failure detection of the 8-bit product without a GPU fault: its kernels' two bounded
waits run out on purpose (barriers that nothing arrives on, a part of the limits), the
flag is reported once, and products before and after are the same."""

import pytest
import torch

from paper_2607_27842_gb300 import featfix as ff

from .test_gpu_ops8 import gemm_inputs, held

pytestmark = pytest.mark.gpu


def test_waits_run_out_and_are_reported(cuda):
    a, sa, w, sw = gemm_inputs(300, 520, 640, 3)
    before, after = held(300, 520, torch.float32), held(300, 520, torch.float32)
    ff.featfix_op_gemm8("f32", a, sa, w, sw, out=before)
    ff.featfix_op_gemm8_watchdog()                       # clean
    limits = ff.featfix_op_gemm8_watchdog_probe()
    # 4 s each: the one by the clock within its polls' spacing, the one by a count of looks
    # within a factor of two
    assert 4.0 <= limits[0] < 4.4 and 2.0 < limits[1] < 8.0, limits
    with pytest.raises(ff.FeatFixError) as e:
        ff.featfix_op_gemm8_watchdog()
    assert e.value.status == ff.ERR_CUDA
    ff.featfix_op_gemm8_watchdog()                       # reported once
    ff.featfix_op_gemm8("f32", a, sa, w, sw, out=after)
    ff.featfix_op_gemm8_watchdog()
    assert torch.equal(before, after)
