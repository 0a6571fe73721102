"""Planning when a query of the runtime fails.  The failure is made on the host: a copy of the test-hooks library, whose
state nobody else has, with its residency queries answered as failed for one call."""
import ctypes
import shutil

import pytest
import torch

from paper_2605_24058_b200 import build, lordba

pytestmark = pytest.mark.gpu


@pytest.fixture()
def fresh(tmp_path):
    path = str(tmp_path / "liblordba_fresh.so")
    shutil.copy(build.build_library(test_hooks=True), path)
    lib = lordba.bind(path)
    lib.lordba_test_fail_queries.restype = ctypes.c_int
    lib.lordba_test_fail_queries.argtypes = [ctypes.c_int]
    return lib


def stream():
    return int(torch.cuda.current_stream().cuda_stream)


def test_a_failed_query_costs_one_call_its_kernel_and_no_later_one(fresh):
    """dx and dW of 8 tokens, whose entries enter as two terms where the streaming kernel runs.  Without the query the call
    still succeeds (in tiles, entries as one term); the next one is what it would have been, bit for bit."""
    T, d, n = 8, 512, 640
    torch.manual_seed(0)
    dh, gate, up = (torch.randn(T, n, device="cuda").to(torch.bfloat16) for _ in range(3))
    x = torch.randn(T, d, device="cuda").to(torch.bfloat16)
    wg, wu = (torch.randn(n, d, device="cuda").to(torch.bfloat16) for _ in range(2))
    want = lordba.gated_backward(dh, gate, up, x, wg, wu)
    got = [torch.full_like(t, 7.0) for t in want]
    g = lordba.GatedGrad(dh=dh.data_ptr(), gate=gate.data_ptr(), up=up.data_ptr(), x=x.data_ptr(), w_gate=wg.data_ptr(), w_up=wu.data_ptr(),
                         dgate=got[0].data_ptr(), dup=got[1].data_ptr(), dx=got[2].data_ptr(), dw_gate=got[3].data_ptr(), dw_up=got[4].data_ptr(),
                         d_in=d, d_hidden=n, ld_dh=n, ld_pre=n, ldx=d, ldw=d, ld_dpre=n, ld_dx=d, ld_dw=d, act=lordba.ACT_SILU)

    def call():
        ws = torch.empty(max(1, fresh.lordba_gated_backward_workspace_bytes(ctypes.byref(g), T)), dtype=torch.uint8, device="cuda")
        rc = fresh.lordba_gated_backward(ctypes.byref(g), T, lordba.BF16, ws.data_ptr(), ws.numel(), stream())
        torch.cuda.synchronize()
        return rc

    fresh.lordba_test_fail_queries(1)
    assert call() == 0
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    dg, du = got[0].double(), got[1].double()
    exact = dg @ wg.double() + du @ wu.double()
    size = dg.abs() @ wg.double().abs() + du.abs() @ wu.double().abs()
    bound = 2 * n * 2.0 ** -23 * size                       # float32 sums of 2 n products, then one rounding
    assert ((got[2].double() - exact).abs() <= bound + 2.0 ** -8 * (exact.abs() + bound)).all()
    fresh.lordba_test_fail_queries(0)
    assert call() == 0
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # a failure after an answer changes nothing
    fresh.lordba_test_fail_queries(1)
    assert call() == 0
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    code = ctypes.c_int(0)
    assert fresh.lordba_device_status(ctypes.byref(code), stream()) == 0


def test_the_product_library_has_no_such_switch():
    assert not hasattr(lordba.load(), "lordba_test_fail_queries")
