"""Tensors of another GPU than the current one are refused by the 8-bit operators'
binding, before anything is launched.  (Stand-ins that only carry a device: one GPU is
enough.)"""

import pytest
import torch

from paper_2607_27842_gb300 import featfix as ff

pytestmark = pytest.mark.gpu


class Elsewhere(torch.Tensor):
    """A tensor without memory that says it is on another device."""

    @classmethod
    def of(cls, size, dtype, device):
        return torch.Tensor._make_wrapper_subclass(cls, size, dtype=dtype, device=device)

    @classmethod
    def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
        raise NotImplementedError(str(func))


def test_tensors_of_another_gpu_are_refused(cuda):
    bf16, u8, f32 = torch.bfloat16, torch.uint8, torch.float32
    sizes = {"x": ((4, 256), bf16), "q": ((4, 256), u8), "s": ((2, 4), f32), "w": ((256, 256), u8), "sw": ((2, 2), f32),
             "pos": ((1, 4), torch.int32), "one": ((256,), bf16)}
    near = {n: torch.zeros(d, dtype=t, device=cuda) for n, (d, t) in sizes.items()}
    far = {n: Elsewhere.of(d, t, "cuda:%d" % (torch.cuda.current_device() + 1)) for n, (d, t) in sizes.items()}
    calls = {
        ("x", "one"): lambda t, o: ff.featfix_op_rms_norm("bf16", t["x"], t["one"], 1e-6, out=o["x"]),
        ("x", "q", "s"): lambda t, o: ff.featfix_op_quant8("bf16", t["x"], t["q"], t["s"]),
        ("q", "s", "w", "sw"): lambda t, o: ff.featfix_op_gemm8("bf16", t["q"], t["s"], t["w"], t["sw"], out=o["x"]),
        ("x", "pos"): lambda t, o: ff.featfix_op_rope("bf16", t["pos"], (128,), 128, q=t["x"], q_out=o["x"])}
    n0 = ff.featfix_launch_count()
    for names, call in calls.items():
        for name in names:
            with pytest.raises(ff.FeatFixError) as e:
                call({**near, name: far[name]}, near)
            assert e.value.status == ff.ERR_INVALID_ARG and "GPU" in str(e.value), (name, str(e.value))
    assert ff.featfix_launch_count() == n0
