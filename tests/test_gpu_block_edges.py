"""Calls of the operators next to the adapters at the edges of what they take: pre-activations that are not finite, very many
columns, tensors that autograd watches."""
import math

import pytest
import torch

from paper_2605_24058_b200 import lordba

pytestmark = pytest.mark.gpu


# 4 rows are streamed, 300 go through tiles
@pytest.mark.parametrize("T", [4, 300])
@pytest.mark.parametrize("act", [lordba.ACT_SILU, lordba.ACT_GELU_TANH])
@pytest.mark.parametrize("dtype,bits", [(torch.float16, 16), (torch.bfloat16, 16), (torch.float16, 8)])
def test_a_gate_of_minus_infinity_is_shut(T, act, dtype, bits):
    """An addend of -inf masks its entry: act(-inf) = 0 and act'(-inf) = 0, forward and backward, and no other entry
    changes.  +inf and NaN go through as the formulas say."""
    n, d = 264, 64
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T + bits)
    x, wg, wu = (torch.randn(r, d, generator=gen, device="cuda").to(dtype) for r in (T, n, n))
    scales = None
    if bits == 8:
        (x, sx), (wg, sg), (wu, su) = (lordba.int8_quantize_rows(t) for t in (x, wg, wu))
        scales = (sx, sg, su)
    add = torch.zeros(T, n, dtype=dtype, device="cuda")
    call = lambda a: lordba.gated_forward(x, wg, wu, act=act, scales=scales, dtype=dtype, gate_add=a, up_add=torch.zeros_like(a), save=True)
    plain, plain_gate, plain_up = call(add)
    masked = add.clone()
    masked[1, 5], masked[2, 263], masked[3, 0], masked[3, 7], masked[0, 100] = -math.inf, -math.inf, math.inf, math.nan, -math.inf
    shut = masked == -math.inf
    h, gate, up = call(masked)
    assert (h[shut] == 0).all() and (gate[shut] == -math.inf).all()
    assert h[3, 0].abs() == math.inf and h[3, 7].isnan()
    same = masked == 0
    assert torch.equal(h[same], plain[same]) and torch.equal(gate[same], plain_gate[same]) and torch.equal(up, plain_up)
    dh = torch.randn(T, n, generator=gen, device="cuda").to(dtype)
    gate[3, 0] = gate[3, 7] = 1.0
    dgate, dup = lordba.gated_backward(dh, gate, up, act=act)[:2]
    assert (dgate[shut] == 0).all() and (dup[shut] == 0).all()
    assert dgate.isfinite().all() and dup.isfinite().all()


@pytest.mark.parametrize("T", [4, 300])
def test_a_stored_gate_that_overflowed_float16_has_no_gradient(T):
    """g = -80000 is -inf in float16; the unrounded forward gives h = 0, and the gradients from the stored value are
    those of a shut gate: dx and dw stay finite."""
    n, d = 72, 16
    x = torch.full((T, d), 100.0, dtype=torch.float16, device="cuda")
    w = torch.full((n, d), 0.01, dtype=torch.float16, device="cuda")
    w[3] = -50.0
    up = torch.full((n, d), 0.01, dtype=torch.float16, device="cuda")
    h, gate, u = lordba.gated_forward(x, w, up, save=True)
    assert (gate[:, 3] == -math.inf).all() and (h[:, 3] == 0).all() and (h[:, 4] > 100).all()
    dh = torch.ones(T, n, dtype=torch.float16, device="cuda")
    dgate, dup, dx, dwg, dwu = lordba.gated_backward(dh, gate, u, x, w, up)
    assert (dgate[:, 3] == 0).all() and (dup[:, 3] == 0).all()
    assert all(t.isfinite().all() for t in (dgate, dup, dx)) and (dwg[3] == 0).all() and (dwu[3] == 0).all()


def test_dx_of_few_tokens_and_very_many_columns():
    """More columns than the streaming kernel's grid holds (65535 tiles of 128): tiles take over, also up to 64 tokens, where
    the gradient's entries otherwise enter as two terms.  dgate and dup are held to the formula elsewhere; dx to the
    float64 product of the returned entries: 2 d_hidden additions of 2^-23, one rounding to bfloat16 (2^-8)."""
    n, d = 8, 65535 * 128 + 8
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    for T in (1, 3, 65):
        dh, gate, up = (torch.randn(T, n, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(3))
        wg, wu = (torch.randn(n, d, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
        dgate, dup, dx, _, _ = lordba.gated_backward(dh, gate, up, None, wg, wu)
        assert lordba.device_status() == 0
        for first in range(0, d, 1 << 20):
            a, b = wg[:, first:first + (1 << 20)].double(), wu[:, first:first + (1 << 20)].double()
            want = dgate.double() @ a + dup.double() @ b
            size = dgate.double().abs() @ a.abs() + dup.double().abs() @ b.abs()
            tol = 2 * n * 2.0 ** -23 * size
            tol = tol + 2.0 ** -8 * (want.abs() + tol)
            assert ((dx[:, first:first + (1 << 20)].double() - want).abs() <= tol).all()


# ------------------------------------------------------------------------------ autograd

def test_calls_do_not_lose_a_gradient_silently():
    """The calls record no graph: with gradients on they refuse tensors that ask for one, as torch's functions with an
    output argument do; without, and on detached tensors, they run."""
    w = torch.randn(32, 64, device="cuda").to(torch.bfloat16)
    x = torch.randn(4, 64, device="cuda").to(torch.bfloat16)
    h = torch.zeros(4, 32, dtype=torch.bfloat16, device="cuda")
    asks = lambda t: t.detach().clone().requires_grad_(True)
    q, s = lordba.int8_quantize_rows(x)
    w8, sw = lordba.int8_quantize_rows(w)
    calls = [lambda f: lordba.gated_forward(f(x), w, w), lambda f: lordba.gated_forward(x, f(w), w), lambda f: lordba.gated_forward(x, w, w, gate_add=h, up_add=f(h)),
             lambda f: lordba.gated_forward(q, w8, w8, scales=(s, f(sw), sw)), lambda f: lordba.gated_backward(h, h, f(h)), lambda f: lordba.dropout(f(x), 0.1, 1),
             lambda f: lordba.dropout(x, 0.1, 1, out=f(x)), lambda f: lordba.int8_quantize_rows(f(x)), lambda f: lordba.int8_linear(q, s, w8, f(sw))]
    for call in calls:
        with pytest.raises(RuntimeError):
            call(asks)
        with torch.no_grad():
            call(asks)
        call(lambda t: t.detach().clone())


def test_writes_into_given_buffers_are_seen_by_autograd():
    """A tensor that autograd keeps and a call overwrites: torch's own check finds it."""
    x = torch.randn(4, 64, device="cuda")
    leaf = torch.randn(4, 64, device="cuda", requires_grad=True)
    y = (leaf * x).sum()
    before = x._version
    lordba.dropout(x, 0.5, 1, out=x)
    assert x._version > before
    with pytest.raises(RuntimeError):
        y.backward()
    b = lambda *shape: torch.zeros(*shape, dtype=torch.bfloat16, device="cuda")
    q8, s4 = torch.zeros(4, 64, dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
    w8, s32 = torch.ones(32, 64, dtype=torch.int8, device="cuda"), torch.ones(32, device="cuda")
    h, g, u, y8 = b(4, 32), b(4, 32), b(4, 32), b(4, 32)
    dg, du, dx, dwg, dwu = b(4, 32), b(4, 32), b(4, 64), b(32, 64), b(32, 64)
    lordba.int8_quantize_rows(b(4, 64), q=q8, scale=s4)
    lordba.int8_linear(q8, s4, w8, s32, y8)
    lordba.gated_forward(b(4, 64), b(32, 64), b(32, 64), h=h, gate=g, up=u)
    lordba.gated_backward(h, g, u, b(4, 64), b(32, 64), b(32, 64), dg, du, dx, dwg, dwu)
    assert all(t._version == 1 for t in (h, g, u, y8, q8, s4, dg, du, dx, dwg, dwu))
    with torch.inference_mode():
        lordba.dropout(torch.ones(4, 8, device="cuda"), 0.5, 1, out=torch.ones(4, 8, device="cuda"))
        kept = torch.ones(4, 8, device="cuda")
    lordba.dropout(torch.ones(4, 8, device="cuda"), 0.5, 1, out=kept)             # an inference tensor has no version


def test_a_type_that_the_result_will_not_have_is_refused():
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(32, 64, dtype=torch.bfloat16, device="cuda")
    assert lordba.gated_forward(x, w, w, dtype=torch.bfloat16)[0].dtype == torch.bfloat16
    with pytest.raises(TypeError):
        lordba.gated_forward(x, w, w, dtype=torch.float16)
    (q, s), (w8, sw) = lordba.int8_quantize_rows(x), lordba.int8_quantize_rows(w)
    h = torch.zeros(4, 32, dtype=torch.float16, device="cuda")
    assert lordba.gated_forward(q, w8, w8, h=h, scales=(s, sw, sw))[0] is h
    with pytest.raises(TypeError):
        lordba.gated_forward(q, w8, w8, h=h, scales=(s, sw, sw), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        lordba.gated_forward(x, w, w, dtype="bfloat16")
