"""The 8-bit operators from several host threads at once."""

import ctypes
import threading
import time

import pytest
import torch

from paper_2607_27842_gb300 import featfix as ff

from .test_gpu_ops8 import check, randn, rms

pytestmark = pytest.mark.gpu


def test_wide_norms_of_two_threads(cuda):
    """Two widths past registers from two host threads at once, each on a stream of its
    own: no call's preparation may be in another's way."""
    lib, calls, bad = ff.lib(), 4000, []
    widths = (20001, 32768)
    xs = [randn((4, C), 30 + i) for i, C in enumerate(widths)]
    outs = [torch.empty_like(x) for x in xs]
    streams = [torch.cuda.Stream() for _ in widths]
    torch.cuda.synchronize()
    start = threading.Barrier(2)

    def work(i):
        C, p, null = widths[i], ctypes.c_void_p, ctypes.c_void_p(None)
        args = (0, 4, C, p(xs[i].data_ptr()), C, null, 0, null, 0, null, ctypes.c_float(1e-6), p(outs[i].data_ptr()), C, null, 0,
                null, 0, p(streams[i].cuda_stream))
        start.wait()
        bad.extend(s for s in (lib.featfix_op_rms_norm(*args) for _ in range(calls)) if s != ff.OK)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not bad, (len(bad), set(bad))
    for x, o, C in zip(xs, outs, widths):
        y = rms(x.double(), None, 1e-6)
        check(o, y, "f32", y.abs() * ((C + 8) * 2.0 ** -25 + 2.0 ** -21))


def test_a_full_launch_queue_leaves_python_to_other_threads(cuda):
    """A launch that waits for room in its stream's queue must not hold the interpreter:
    while one thread launches behind a kernel of a second, this one goes on."""
    x = randn((4, 256), 40)
    q, s = torch.empty((4, 256), dtype=torch.uint8, device=cuda), torch.empty((2, 4), device=cuda)
    stream, done = torch.cuda.Stream(), threading.Event()
    ff.featfix_op_quant8("f32", x, q, s)
    torch.cuda.synchronize()

    def work():
        with torch.cuda.stream(stream):
            torch.cuda._sleep(2_000_000_000)          # about a second
            for _ in range(6000):
                ff.featfix_op_quant8("f32", x, q, s)
        done.set()

    t = threading.Thread(target=work)
    t.start()
    gap, last, began = 0.0, time.monotonic(), time.monotonic()
    while not done.is_set() and time.monotonic() - began < 20:
        time.sleep(0.002)
        now = time.monotonic()
        gap, last = max(gap, now - last), now
    t.join()
    took = time.monotonic() - began
    torch.cuda.synchronize()
    assert took > 0.5, took                            # the queue was full: its thread had to wait
    assert gap < 0.25, gap
