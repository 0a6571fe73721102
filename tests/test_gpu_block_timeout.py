"""Waits that run out in the product kernels (see test_gpu_timeout.py for the method: a library built with
shorter limits and a hook that leaves out one stage's copies; nothing faults or hangs).  Checked for the tile
kernel, the streaming kernel and its form for unaligned operands: the call itself succeeds, the status is
reported once, the output keeps its old values, and the next call is correct."""
import ctypes

import pytest
import torch

from paper_2605_24058_b200 import build, lordba

pytestmark = pytest.mark.gpu

ETIMEOUT = 5


@pytest.fixture(scope="module")
def hooks():
    lib = lordba.bind(build.build_library(test_hooks=True))
    lib.lordba_test_skip_item.restype = ctypes.c_int
    lib.lordba_test_skip_item.argtypes = [ctypes.c_int]
    yield lib
    lib.lordba_test_skip_item(-1)


# many rows: tiles; few rows: streamed weights, split over a cluster; an odd pitch: the unaligned form
@pytest.mark.parametrize("T,d_in,pitch,d_out", [(1024, 1024, 1024, 2048), (8, 2048, 2048, 512), (8, 2048, 2049, 512)])
@pytest.mark.parametrize("skip", [0, 1])
def test_a_wait_that_runs_out_is_reported_and_nothing_is_written(hooks, T, d_in, pitch, d_out, skip):
    one = lambda n: torch.ones(n, device="cuda")
    x = torch.randint(-127, 128, (T, d_in), dtype=torch.int8, device="cuda")
    w = torch.randint(-127, 128, (d_out, pitch), dtype=torch.int8, device="cuda")[:, :d_in]
    s_x, s_w = one(T), one(d_out)
    y = torch.full((T, d_out), 7.0, device="cuda")
    p = lordba.Int8Proj(x.data_ptr(), s_x.data_ptr(), w.data_ptr(), s_w.data_ptr(), y.data_ptr(), d_in, d_out, d_in, pitch, d_out)
    stream = int(torch.cuda.current_stream().cuda_stream)
    ws = torch.empty(max(1, hooks.lordba_int8_linear_workspace_bytes(ctypes.byref(p), T)), dtype=torch.uint8, device="cuda")

    def call():
        return hooks.lordba_int8_linear(ctypes.byref(p), T, lordba.F32, ws.data_ptr(), ws.numel(), stream)

    def status():
        code = ctypes.c_int(0)
        return hooks.lordba_device_status(ctypes.byref(code), stream), code.value

    assert status() == (0, 0)
    hooks.lordba_test_skip_item(skip)
    assert call() == 0
    rc, code = status()
    assert rc == ETIMEOUT and code in (1, 2, 3, 4)
    assert status() == (0, 0)
    assert (y == 7.0).all()
    hooks.lordba_test_skip_item(-1)
    assert call() == 0
    assert status() == (0, 0)
    # exact in float64, and the kernel's float32 of an integer below 2^31 is its nearest
    assert torch.equal(y, (x.double() @ w.double().t()).float())
