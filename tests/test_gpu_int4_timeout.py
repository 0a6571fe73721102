"""Waits that run out in the kernel that widens 4-bit weights on their way (see test_gpu_timeout.py for the method: a library
built with shorter limits and a hook that leaves out one stage's copy; nothing faults or hangs)."""
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


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("skip", [0, 1])
def test_a_wait_that_runs_out_is_reported_and_nothing_is_written(hooks, backward, skip):
    T, d_in, d_out = 64, 2048, 1024
    f = hooks.lordba_int4_linear_backward if backward else hooks.lordba_int4_linear
    n_in, n_out = (d_out, d_in) if backward else (d_in, d_out)
    u = torch.randint(0, 16, (d_out, d_in), dtype=torch.uint8, device="cuda")
    q = lordba.int4_pack(u)
    scale = torch.full((d_out, d_in // 128), 0.5, dtype=torch.bfloat16, device="cuda")
    x = torch.randint(-3, 4, (T, n_in), device="cuda").to(torch.bfloat16)
    y = torch.full((T, n_out), 7.0, dtype=torch.bfloat16, device="cuda")
    p = lordba.Int4Proj(x.data_ptr(), y.data_ptr(), q.data_ptr(), scale.data_ptr(), 0, d_in, d_out, n_in, n_out, q.stride(0), scale.stride(0), 0, 128, 0)
    stream = int(torch.cuda.current_stream().cuda_stream)
    call = lambda: f(ctypes.byref(p), T, lordba.BF16, None, 0, stream)

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
    # integers and halves: exact in bfloat16 operands and float32 sums, rounded once
    w = 0.5 * (u.double() - 8)
    assert torch.equal(y, (x.double() @ (w if backward else w.t())).to(torch.bfloat16))
