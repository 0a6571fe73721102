"""GPU parity of the operators next to the adapters (8-bit base projection, gated feed-forward block with its
gradients, dropout) against plain float64 implementations written here.

Tolerances, from the arithmetic.  u is the unit roundoff of the output type (bf16 2^-8, f16 2^-11, f32 2^-24;
f16 results below 2^-14 are multiples of 2^-24).
  8-bit product: the integer sum is exact; three float32 roundings follow, then u.
  16-bit products: each of the K additions of a float32 sum may lose 2^-23 of the sum of magnitudes
    (truncating adders), so |err| <= K 2^-23 sum |a b|, then u.
  activation: the hardware exponential and division are good to 2^-20 for |g| < 16; 2^-18 covers both.
  gradients to x and to the weights are held to the float64 products of the dgate / dup that the call itself
    returned (they are operands of the products in that type), dgate and dup to the formula.  Up to 64 tokens
    the products take dgate and dup as two terms, and are held to products of the formula's values: the second
    term leaves u^2 of an entry (of float16 at least 2^-25), the formula 2^-18 of its magnitudes.
"""
import math

import numpy as np
import pytest
import torch

from paper_2605_24058_b200 import lordba

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
TINY = {"bf16": 0.0, "f16": 2.0 ** -25, "f32": 0.0}


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def matrix(rng, rows, cols, dtype, pad=0, scale=1.0, lead=0):
    """(device view, float64 values) of rows x cols draws; pad extra columns after each row, lead elements before the first."""
    buf = torch.from_numpy(rng.standard_normal(rows * (cols + pad) + lead).astype(np.float32) * np.float32(scale)).to(TYPES[dtype])
    t = buf.cuda()[lead:].view(rows, cols + pad)[:, :cols]
    return t, f64(t)


def int8_matrix(rng, rows, cols, pad=0, lead=0, low=-127):
    buf = torch.from_numpy(rng.integers(low, 128, rows * (cols + pad) + lead, dtype=np.int8))
    t = buf.cuda()[lead:].view(rows, cols + pad)[:, :cols]
    return t, t.cpu().numpy().astype(np.float64)


def scales(rng, n):
    s = torch.from_numpy(np.exp(rng.standard_normal(n) * 0.5).astype(np.float32)).cuda()
    return s, f64(s)


def target(rows, cols, dtype, pad=0, lead=0):
    """An output buffer full of sentinels, and its rows x cols view."""
    buf = torch.full((rows * (cols + pad) + lead,), 77.0, dtype=TYPES[dtype], device="cuda")
    return buf, buf[lead:].view(rows, cols + pad)[:, :cols]


def untouched(buf, rows, cols, pad, lead):
    v = f64(buf)
    assert (v[:lead] == 77).all()
    assert pad == 0 or (v[lead:].reshape(rows, cols + pad)[:, cols:] == 77).all(), "the padding of a row was written"


def close(got, want, bound, dtype, what):
    got = f64(got)
    assert got.shape == want.shape
    tol = bound + UNIT[dtype] * (np.abs(want) + bound) + TINY[dtype]
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), "%s: %d of %d off, first at %s: got %r want %r tol %r" % (
        what, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0], tol[bad][0])


def clean():
    assert lordba.device_status() == 0


# ------------------------------------------------------------------------------------------ quantisation

@pytest.mark.parametrize("T,d,pad,lead", [(1, 1, 0, 0), (1, 4096, 0, 0), (3, 7, 0, 0), (9, 1024, 8, 0), (5, 1025, 0, 0), (17, 1000, 3, 1),
                                          (64, 4096, 0, 0), (3, 11008, 0, 0), (2, 12289, 5, 3), (2, 30001, 0, 0), (2, 16384, 0, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_quantize_rows(T, d, pad, lead, dtype):
    rng = np.random.default_rng(d * 7 + T)
    x, v = matrix(rng, T, d, dtype, pad, 3.0, lead)
    q, s = lordba.int8_quantize_rows(x)
    v32 = v.astype(np.float32)
    amax = np.abs(v32).max(axis=1, keepdims=True)
    assert np.array_equal(s.cpu().numpy(), (amax / np.float32(127))[:, 0])
    want = np.rint(v32 * (np.float32(127) / amax)).astype(np.int8)
    assert np.array_equal(q.cpu().numpy(), want)
    assert np.abs(want).max() == 127
    # a caller's q with an odd pitch
    buf = torch.full((T, d + 3), 99, dtype=torch.int8, device="cuda")
    lordba.int8_quantize_rows(x, q=buf[:, :d], scale=s)
    assert np.array_equal(buf.cpu().numpy()[:, :d], want) and (buf[:, d:] == 99).all()


@pytest.mark.parametrize("d", [40, 1500])
def test_quantize_rows_without_a_number_to_scale_by(d):
    x = torch.randn(6, d, device="cuda")
    x[1] = 0.0
    x[2, d // 2] = math.inf
    x[3, d - 1] = math.nan
    x[4] *= 1e-37                         # below 2^-120
    x[5, 0] = -math.inf
    x[5, 1] = math.nan
    q, s = lordba.int8_quantize_rows(x)
    s = s.cpu().numpy()
    assert s[0] > 0 and s[1] == 0 and s[4] == 0 and np.isnan(s[[2, 3, 5]]).all()
    assert (q[1:].cpu().numpy() == 0).all()
    # the product: NaN rows stay rows
    w = torch.ones(8, d, dtype=torch.int8, device="cuda")
    y = lordba.int8_linear(q, torch.from_numpy(s).cuda(), w, torch.ones(8, device="cuda"), dtype=torch.float32).cpu().numpy()
    assert np.isnan(y[[2, 3, 5]]).all() and np.isfinite(y[[0, 1, 4]]).all() and (y[[1, 4]] == 0).all()


# --------------------------------------------------------------------------------------- the 8-bit product

INT8_SIZES = [  # T, d_in, d_out, padx, padw, pady, lead
    (1, 1, 1, 0, 0, 0, 0), (1, 16, 8, 0, 0, 0, 0), (1, 4096, 1000, 0, 0, 0, 0), (2, 128, 128, 0, 0, 0, 0), (5, 129, 131, 0, 0, 0, 0),
    (8, 2048, 640, 0, 0, 0, 0), (16, 1000, 257, 8, 24, 1, 0), (17, 4096, 384, 0, 0, 0, 0), (33, 256, 96, 16, 0, 8, 0),
    (64, 1111, 333, 0, 0, 0, 0), (65, 640, 512, 0, 0, 0, 0), (128, 2048, 1024, 0, 0, 0, 0), (129, 160, 2049, 0, 0, 0, 0),
    (256, 512, 256, 0, 0, 0, 0), (300, 1001, 700, 7, 0, 3, 1), (513, 384, 520, 0, 16, 0, 0), (777, 96, 1533, 0, 0, 0, 5),
    (1025, 1024, 1024, 0, 0, 0, 0), (2048, 64, 4096, 0, 0, 0, 0), (2500, 300, 600, 4, 4, 4, 0),
    (600, 256, 1533, 0, 0, 3, 0), (700, 128, 2045, 0, 0, 3, 0)]


@pytest.mark.parametrize("T,d_in,d_out,padx,padw,pady,lead", INT8_SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_int8_linear(T, d_in, d_out, padx, padw, pady, lead, dtype):
    rng = np.random.default_rng(T * 31 + d_in)
    x, vx = int8_matrix(rng, T, d_in, padx, lead)
    w, vw = int8_matrix(rng, d_out, d_in, padw, lead)
    s_x, vsx = scales(rng, T)
    s_w, vsw = scales(rng, d_out)
    buf, y = target(T, d_out, dtype, pady, lead)
    assert lordba.int8_linear(x, s_x, w, s_w, y) is y
    clean()
    want = (vx @ vw.T) * vsx[:, None] * vsw
    close(y, want, 4 * 2.0 ** -24 * np.abs(want), dtype, "y")
    untouched(buf, T, d_out, pady, lead)


def test_int8_linear_float16_and_new_output():
    rng = np.random.default_rng(0)
    x, vx = int8_matrix(rng, 70, 500, low=-128)
    w, vw = int8_matrix(rng, 90, 500, low=-128)
    s_x, s_w = torch.full((70,), 2.0 ** -10, device="cuda"), torch.full((90,), 2.0 ** -6, device="cuda")
    y = lordba.int8_linear(x, s_x, w, s_w, dtype=torch.float16)
    want = (vx @ vw.T) * 2.0 ** -16
    assert y.dtype == torch.float16
    close(y, want, 4 * 2.0 ** -24 * np.abs(want), "f16", "y")


@pytest.mark.parametrize("T", [3, 200])
def test_int8_sums_are_exact_where_floats_are_not(T):
    """The longest contraction that is taken, all products of one sign: the sum needs 31 bits."""
    K = lordba.INT8_MAX_DIN
    x = torch.full((T, K), -128, dtype=torch.int8, device="cuda")
    w = torch.full((64, K), -128, dtype=torch.int8, device="cuda")
    w[1, 0], w[2] = 127, 127
    one = lambda n: torch.ones(n, device="cuda")
    y = lordba.int8_linear(x, one(T), w, one(64), dtype=torch.float32)
    want = np.full((T, 64), K * 16384.0)
    want[:, 1] -= 255 * 128
    want[:, 2] = -K * 128 * 127.0
    assert np.array_equal(f64(y), want.astype(np.float32).astype(np.float64))


# ------------------------------------------------------------------------------------------- the gated block

def activation(g, act):
    """Value and derivative in float64."""
    if act == lordba.ACT_SILU:
        s = 1 / (1 + np.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    c = math.sqrt(2 / math.pi)
    t = np.tanh(c * (g + 0.044715 * g ** 3))
    return g * (1 + t) / 2, (1 + t) / 2 + g * (1 - t * t) / 2 * c * (1 + 3 * 0.044715 * g * g)


def gated_bounds(vx, vg, vu, g, u, act, scale=None):
    """|err| of g, u and h before the last rounding."""
    K = vx.shape[1]
    if scale is None:
        eg, eu = (K * 2.0 ** -23 * (np.abs(vx) @ np.abs(w).T) + 2.0 ** -23 * np.abs(p) for w, p in ((vg, g), (vu, u)))
    else:
        eg, eu = (6 * 2.0 ** -24 * np.abs(p) + 2.0 ** -24 * scale for p in (g, u))
    a = activation(g, act)[0]
    # |act'| <= 1.13; the two errors meet in the product as well
    eh = 1.13 * eg * (np.abs(u) + eu) + np.abs(a) * eu + 2.0 ** -18 * np.abs(a * u)
    return eg, eu, eh


GATED_SIZES = [  # T, d_in, d_hidden, pad, lead
    (1, 1, 1, 0, 0), (1, 64, 64, 0, 0), (1, 2048, 700, 0, 0), (2, 128, 128, 0, 0), (8, 512, 1000, 0, 0), (9, 100, 131, 0, 0), (16, 320, 256, 8, 0),
    (17, 77, 333, 5, 1), (40, 1024, 130, 0, 0), (64, 256, 512, 0, 0), (65, 64, 129, 0, 3), (128, 640, 384, 0, 0), (150, 500, 300, 0, 0),
    (256, 128, 256, 64, 0), (333, 520, 1365, 0, 0), (600, 192, 640, 0, 0), (1100, 256, 520, 0, 0), (600, 192, 635, 5, 0), (900, 64, 2043, 5, 0)]


@pytest.mark.parametrize("T,d_in,d_hidden,pad,lead", GATED_SIZES)
@pytest.mark.parametrize("dtype,act,add,save", [("bf16", 0, False, False), ("f16", 1, True, True), ("bf16", 1, False, True), ("f16", 0, True, False)])
def test_gated_forward(T, d_in, d_hidden, pad, lead, dtype, act, add, save):
    rng = np.random.default_rng(T * 13 + d_hidden)
    x, vx = matrix(rng, T, d_in, dtype, pad, 1.0, lead)
    wg, vg = matrix(rng, d_hidden, d_in, dtype, pad, 1.5 / math.sqrt(d_in), lead)
    wu, vu = matrix(rng, d_hidden, d_in, dtype, pad, 1.5 / math.sqrt(d_in), lead)
    ga, vga = matrix(rng, T, d_hidden, dtype, pad, 0.5, lead)
    ua, vua = matrix(rng, T, d_hidden, dtype, pad, 0.5, lead)
    g, u = vx @ vg.T, vx @ vu.T
    if add:
        g, u = g + vga, u + vua
    buf, h = target(T, d_hidden, dtype, pad, lead)
    got, gate, up = lordba.gated_forward(x, wg, wu, h=h, act=act, gate_add=ga if add else None, up_add=ua if add else None, save=save)
    clean()
    assert got is h and (gate is not None) == save
    eg, eu, eh = gated_bounds(vx, vg, vu, g, u, act)
    close(h, activation(g, act)[0] * u, eh, dtype, "h")
    untouched(buf, T, d_hidden, pad, lead)
    if save:
        close(gate, g, eg, dtype, "gate")
        close(up, u, eu, dtype, "up")


@pytest.mark.parametrize("T,d_in,d_hidden,pad,lead", GATED_SIZES)
@pytest.mark.parametrize("dtype,act,add,save", [("bf16", 0, False, False), ("f16", 1, True, True)])
def test_gated_forward_int8(T, d_in, d_hidden, pad, lead, dtype, act, add, save):
    rng = np.random.default_rng(T * 17 + d_hidden)
    x, vx = int8_matrix(rng, T, d_in, pad, lead)
    wg, vg = int8_matrix(rng, d_hidden, d_in, pad, lead)
    wu, vu = int8_matrix(rng, d_hidden, d_in, pad, lead)
    s = 1 / (74.0 * 74.0 * math.sqrt(d_in))
    (sx, vsx), (sg, _), (su, _) = scales(rng, T), scales(rng, d_hidden), scales(rng, d_hidden)
    sg, su = sg * s, su * s
    ga, vga = matrix(rng, T, d_hidden, dtype, pad, 0.5, lead)
    ua, vua = matrix(rng, T, d_hidden, dtype, pad, 0.5, lead)
    g, u = (vx @ vg.T) * vsx[:, None] * f64(sg), (vx @ vu.T) * vsx[:, None] * f64(su)
    size = np.maximum(np.abs(g), np.abs(u))
    if add:
        g, u = g + vga, u + vua
    h, gate, up = lordba.gated_forward(x, wg, wu, act=act, scales=(sx, sg, su), dtype=TYPES[dtype], gate_add=ga if add else None,
                                       up_add=ua if add else None, save=save)
    clean()
    eg, eu, eh = gated_bounds(vx, vg, vu, g, u, act, scale=8 * size)
    close(h, activation(g, act)[0] * u, eh, dtype, "h")
    if save:
        close(gate, g, eg, dtype, "gate")
        close(up, u, eu, dtype, "up")


def test_gated_forward_in_joint_buffers():
    """gate and up as the halves of one buffer that held the addends: read, then overwritten in place."""
    rng = np.random.default_rng(5)
    T, d_in, n = 140, 192, 264
    x, vx = matrix(rng, T, d_in, "bf16")
    w, vw = matrix(rng, n, 2 * d_in, "bf16", 0, 0.1)                   # the two weights side by side
    both, vb = matrix(rng, T, 2 * n, "bf16")
    vgu = [vx @ vw[:, :d_in].T + vb[:, :n], vx @ vw[:, d_in:].T + vb[:, n:]]
    gate, up = both[:, :n], both[:, n:]
    wg, wu = w[:, :d_in], w[:, d_in:]
    h, _, _ = lordba.gated_forward(x, wg, wu, gate_add=gate, up_add=up, gate=gate, up=up)
    eg, eu, eh = gated_bounds(vx, vw[:, :d_in], vw[:, d_in:], *vgu, 0)
    close(gate, vgu[0], eg, "bf16", "gate")
    close(up, vgu[1], eu, "bf16", "up")
    close(h, activation(vgu[0], 0)[0] * vgu[1], eh, "bf16", "h")


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("T", [4, 200])
def test_gated_forward_far_out(act, T):
    """Large pre-activations: the gate is 0 or g itself; a NaN or an infinity stays in its row and column."""
    x = torch.zeros(T, 16, dtype=torch.bfloat16, device="cuda")
    x[0, 0], x[1, 0], x[2, 1], x[3, 2] = 1000.0, -1000.0, math.nan, math.inf
    w = torch.zeros(32, 16, dtype=torch.bfloat16, device="cuda")
    w[:, 0], w[0, 1], w[1, 2] = 1.0, 1.0, 1.0
    one = torch.zeros(32, 16, dtype=torch.bfloat16, device="cuda")
    one[:, 0] = 1.0
    h = f64(lordba.gated_forward(x, w, one, act=act)[0])
    assert (h[0] == 1e6 - 1e6 % 2 ** 12).all() or np.allclose(h[0], 1e6, rtol=2 ** -8)
    assert (h[1] == 0).all()
    assert np.isnan(h[2]).all() and np.isnan(h[3]).all()             # NaN * 0 and inf * 0 in every column's sum
    assert (h[4:] == 0).all()


# ------------------------------------------------------------------------------------------ the gradients

GRAD_SIZES = [  # T, d_in, d_hidden, pad, lead
    (1, 1, 1, 0, 0), (1, 512, 640, 0, 0), (2, 64, 128, 0, 0), (7, 100, 130, 0, 0), (16, 256, 1024, 8, 0), (33, 129, 257, 0, 1), (64, 512, 384, 0, 0),
    (65, 72, 264, 0, 0), (128, 256, 256, 0, 0), (200, 333, 700, 3, 0), (333, 520, 1365, 0, 0), (700, 1024, 256, 0, 0), (2500, 96, 200, 0, 0), (3000, 130, 72, 5, 0), (4097, 256, 130, 0, 0)]


@pytest.mark.parametrize("T,d_in,d_hidden,pad,lead", GRAD_SIZES)
@pytest.mark.parametrize("dtype,act", [("bf16", 0), ("f16", 1)])
def test_gated_backward(T, d_in, d_hidden, pad, lead, dtype, act):
    rng = np.random.default_rng(T * 19 + d_hidden)
    x, vx = matrix(rng, T, d_in, dtype, pad, 1.0, lead)
    wg, vg = matrix(rng, d_hidden, d_in, dtype, pad, 1 / math.sqrt(d_in), lead)
    wu, vu = matrix(rng, d_hidden, d_in, dtype, pad, 1 / math.sqrt(d_in), lead)
    (gate, g), (up, u), (dh, v) = (matrix(rng, T, d_hidden, dtype, pad, 1.0, lead) for _ in range(3))
    bufs = [target(T, d_hidden, dtype, pad, lead) for _ in range(2)] + [target(T, d_in, dtype, pad, lead)] + [
        target(d_hidden, d_in, dtype, pad, lead) for _ in range(2)]
    dgate, dup, dx, dwg, dwu = (b[1] for b in bufs)
    lordba.gated_backward(dh, gate, up, x, wg, wu, dgate, dup, dx, dwg, dwu, act=act)
    clean()
    a, slope = activation(g, act)
    # slope = f + g f (1 - f) k': both terms to 2^-18 of themselves; |g f (1 - f) k'| <= 1.2
    close(dgate, v * u * slope, 2.0 ** -18 * np.abs(v * u) * 2.4, dtype, "dgate")
    close(dup, v * a, 2.0 ** -18 * np.abs(v * a), dtype, "dup")
    dg, du = f64(dgate), f64(dup)
    eg = eu = 0.0
    terms = 1
    if T <= 64:
        dg, du, terms = v * u * slope, v * a, 2
        eg = 2.0 ** -18 * np.abs(v * u) * 2.4 + UNIT[dtype] ** 2 * np.abs(dg) + TINY[dtype]
        eu = 2.0 ** -18 * np.abs(du) + UNIT[dtype] ** 2 * np.abs(du) + TINY[dtype]
    mg, mu = np.abs(dg) + eg, np.abs(du) + eu
    err = terms * 2 * d_hidden * 2.0 ** -23 * (mg @ np.abs(vg) + mu @ np.abs(vu))
    close(dx, dg @ vg + du @ vu, err + (eg + 0 * dg) @ np.abs(vg) + (eu + 0 * du) @ np.abs(vu), dtype, "dx")
    close(dwg, dg.T @ vx, terms * T * 2.0 ** -23 * (mg.T @ np.abs(vx)) + (eg + 0 * dg).T @ np.abs(vx), dtype, "dw_gate")
    close(dwu, du.T @ vx, terms * T * 2.0 ** -23 * (mu.T @ np.abs(vx)) + (eu + 0 * du).T @ np.abs(vx), dtype, "dw_up")
    for (buf, _), rows, cols in zip(bufs, (T, T, T, d_hidden, d_hidden), (d_hidden, d_hidden, d_in, d_in, d_in)):
        untouched(buf, rows, cols, pad, lead)
    # the parts alone give the same bits (into buffers of the same layout: another one may take another kernel)
    again = lambda rows, cols: target(rows, cols, dtype, pad, lead)[1]
    only = lordba.gated_backward(dh, gate, up, None, wg, wu, again(T, d_hidden), again(T, d_hidden), again(T, d_in), act=act)
    assert only[3] is None and torch.equal(only[0], dgate) and torch.equal(only[1], dup) and torch.equal(only[2], dx)
    only = lordba.gated_backward(dh, gate, up, x, None, None, again(T, d_hidden), again(T, d_hidden), None, again(d_hidden, d_in),
                                 again(d_hidden, d_in), act=act)
    assert only[2] is None and torch.equal(only[3], dwg) and torch.equal(only[4], dwu)


@pytest.mark.parametrize("act", [0, 1])
def test_gated_backward_against_differences(act):
    """Central differences of the float64 loss sum(dh act(g) u) at the stored g and u, in single coordinates."""
    rng = np.random.default_rng(11 + act)
    T, d_in, n = 24, 40, 56
    x, vx = matrix(rng, T, d_in, "f16")
    wg, vg = matrix(rng, n, d_in, "f16", 0, 0.2)
    wu, vu = matrix(rng, n, d_in, "f16", 0, 0.2)
    (gate, g), (up, u), (dh, v) = (matrix(rng, T, n, "f16") for _ in range(3))
    dgate, dup, dx, dwg, dwu = (f64(t) for t in lordba.gated_backward(dh, gate, up, x, wg, wu, act=act))
    loss = lambda g, u: float((v * activation(g, act)[0] * u).sum())
    eps = 1e-5

    def slope(dg, du):
        return (loss(g + eps * dg, u + eps * du) - loss(g - eps * dg, u - eps * du)) / (2 * eps)

    zero = np.zeros((T, n))
    for _ in range(12):
        t, i, k = rng.integers(T), rng.integers(n), rng.integers(d_in)
        unit = zero.copy()
        unit[t, i] = 1.0
        row = zero.copy()
        row[t] = 1.0
        col = zero.copy()
        col[:, i] = vx[:, k]
        # one f16 rounding of the result, one of each of the operands' entries (in quadrature at most, summed here)
        spread = lambda *parts: 2 * UNIT["f16"] * sum(np.abs(p).sum() for p in parts) + 1e-6
        assert abs(dgate[t, i] - slope(unit, zero)) <= spread(dgate[t, i])
        assert abs(dup[t, i] - slope(zero, unit)) <= spread(dup[t, i])
        assert abs(dx[t, k] - slope(row * vg[:, k], row * vu[:, k])) <= spread(dgate[t] * vg[:, k], dup[t] * vu[:, k])
        assert abs(dwg[i, k] - slope(col, zero)) <= spread(dgate[:, i] * vx[:, k])
        assert abs(dwu[i, k] - slope(zero, col)) <= spread(dup[:, i] * vx[:, k])


def test_gated_backward_far_out_and_empty():
    dh = torch.ones(2, 8, dtype=torch.float16, device="cuda")
    gate = torch.tensor([[60000, -60000, 300, -300, math.inf, 0, 20, -20.0]] * 2, dtype=torch.float16, device="cuda")
    for act in (0, 1):
        dgate, dup = lordba.gated_backward(dh, gate, dh, act=act)[:2]
        assert dgate[0].tolist()[:6] == [1, 0, 1, 0, 1, 0.5] and dup[0].tolist()[:4] == [60000, 0, 300, 0]
    empty = torch.empty(0, 8, dtype=torch.float16, device="cuda")
    dw = [torch.full((8, 5), 3.0, dtype=torch.float16, device="cuda") for _ in range(2)]
    x0 = torch.empty(0, 5, dtype=torch.float16, device="cuda")
    lordba.gated_backward(empty, empty, empty, x0, dw_gate=dw[0], dw_up=dw[1])
    assert (dw[0] == 0).all() and (dw[1] == 0).all()              # sums over no token
    assert lordba.gated_forward(x0, dw[0], dw[1])[0].shape == (0, 8)
    assert lordba.dropout(empty, 0.5, 1).shape == (0, 8)


# ------------------------------------------------------------------------------------------------- dropout

def philox(c, k):
    """Philox4x32-10 on arrays of uint64 words below 2^32."""
    c, k = [np.asarray(v, np.uint64) for v in c], [int(v) for v in k]
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> half) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> half) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def numbers(T, d, seed, offset):
    groups = (d + 7) // 8
    col, row = np.meshgrid(np.arange(groups), np.arange(T))
    full = lambda v: np.full((T, groups), v, np.uint64)
    w = philox([col, row, full(offset % 2 ** 32), full(offset >> 32)], [seed % 2 ** 32, seed >> 32])
    out = np.empty((T, groups, 8), np.int64)
    for i in range(8):
        out[:, :, i] = (w[i // 2] >> np.uint64(16 * (i % 2))) & np.uint64(0xFFFF)
    return out.reshape(T, -1)[:, :d]


def test_generator_has_the_published_answers():
    """Known answers of Philox4x32-10: zeros, and all ones."""
    assert [int(v) for v in philox([0, 0, 0, 0], [0, 0])] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 2 ** 32 - 1
    assert [int(v) for v in philox([ones] * 4, [ones] * 2)] == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


@pytest.mark.parametrize("T,d,pad,lead", [(1, 1, 0, 0), (1, 4096, 0, 0), (7, 1021, 3, 0), (33, 64, 0, 0), (300, 200, 8, 0), (5, 2049, 0, 1), (3000, 72, 0, 0),
                                          (64, 11008, 0, 0)])
@pytest.mark.parametrize("dtype,p,residual", [("bf16", 0.1, True), ("f16", 0.5, False), ("f32", 0.05, True), ("f32", 0.0, False), ("bf16", 1.0, True)])
def test_dropout(T, d, pad, lead, dtype, p, residual):
    rng = np.random.default_rng(T + d)
    x, v = matrix(rng, T, d, dtype, pad, 1.0, lead)
    r, vr = matrix(rng, T, d, dtype, pad, 1.0, lead)
    seed, offset = 0xFEDCBA9876543210, 0x123456789A
    cut = int(round(p * 65536))
    keep = numbers(T, d, seed, offset) >= cut
    kept = np.where(keep, v * (65536 / max(1, 65536 - cut)), 0.0)
    want = kept + vr if residual else kept
    buf, out = target(T, d, dtype, pad, lead)
    assert lordba.dropout(x, p, seed, offset, residual=r if residual else None, out=out) is out
    close(out, want, 2.0 ** -23 * (np.abs(kept) + np.abs(want)), dtype, "out")
    untouched(buf, T, d, pad, lead)
    if not residual:
        assert np.array_equal(f64(out) == 0, ~keep | (v == 0))
    # in place, over x and over the residual
    for over in (x, r) if residual else (x,):
        a = over.clone() if over.is_contiguous() else over
        again = lordba.dropout(a if over is x else x, p, seed, offset, residual=(a if over is r else r) if residual else None, out=a)
        assert torch.equal(again, out)
        if over is x and residual:
            x = matrix(np.random.default_rng(T + d), T, d, dtype, pad, 1.0, lead)[0]


def test_dropout_drops_what_is_not_finite_and_rate():
    x = torch.full((64, 4096), math.inf, device="cuda")
    y = lordba.dropout(x, 0.25, 3)
    dropped = (y == 0).float().mean().item()
    assert not y.isnan().any() and ((y == 0) | (y == math.inf)).all()
    assert abs(dropped - 0.25) < 6 * math.sqrt(0.25 * 0.75 / x.numel())          # six standard deviations
    assert not torch.equal(y, lordba.dropout(x, 0.25, 4)) and not torch.equal(y, lordba.dropout(x, 0.25, 3, 1))
    assert torch.equal(y, lordba.dropout(x, 0.25, 3))


# ---------------------------------------------------------------------------- streams, order, refusals

def test_calls_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(9)
    x, _ = matrix(rng, 48, 320, "bf16")
    wg, _ = matrix(rng, 200, 320, "bf16", 0, 0.05)
    wu, _ = matrix(rng, 200, 320, "bf16", 0, 0.05)
    dh, _ = matrix(rng, 48, 200, "bf16")

    def all_of(stream=None):
        q, s = lordba.int8_quantize_rows(x, stream=stream)
        w8, sw = lordba.int8_quantize_rows(wg, stream=stream)
        y = lordba.int8_linear(q, s, w8, sw, stream=stream)
        h, g, u = lordba.gated_forward(x, wg, wu, save=True, stream=stream)
        return [y, h, lordba.dropout(h, 0.1, 7, residual=y, stream=stream), *lordba.gated_backward(dh, g, u, x, wg, wu, stream=stream)]

    want = [t.clone() for t in all_of()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = all_of(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = all_of()
    for t in captured:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(captured, want))
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(all_of(), want))           # the same bits every time


def test_the_binding_refuses_what_it_cannot_take():
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(32, 64, dtype=torch.bfloat16, device="cuda")
    q, s = lordba.int8_quantize_rows(x)
    w8, sw = lordba.int8_quantize_rows(w)
    with pytest.raises(ValueError):
        lordba.int8_quantize_rows(x.cpu())
    with pytest.raises(ValueError):
        lordba.int8_quantize_rows(x.t())
    with pytest.raises(TypeError):
        lordba.int8_quantize_rows(x.to(torch.int32))
    with pytest.raises(TypeError):
        lordba.int8_linear(x, s, w8, sw)
    with pytest.raises(ValueError):
        lordba.int8_linear(q, s, w8[:, :32], sw)
    with pytest.raises(TypeError):
        lordba.int8_linear(q, s[:2], w8, sw)
    with pytest.raises(ValueError):
        lordba.int8_linear(q, s, w8, sw, y=torch.zeros(4, 31, device="cuda"))
    with pytest.raises(ValueError):
        lordba.gated_forward(x, w, w, gate_add=x)
    with pytest.raises(ValueError):
        lordba.gated_forward(q, w8, w8)
    with pytest.raises(TypeError):
        lordba.gated_forward(x, w, w.half())
    with pytest.raises(lordba.LordbaError):
        lordba.gated_forward(x.float(), w.float(), w.float())
    with pytest.raises(lordba.LordbaError):
        lordba.gated_forward(x, w, w, act=5)
    h = torch.zeros(4, 32, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(lordba.LordbaError):
        lordba.gated_forward(x, w, w, gate=h, up=h)                            # one buffer for both
    with pytest.raises(ValueError):
        lordba.gated_backward(h, h, h, dx=x)
    with pytest.raises(lordba.LordbaError):
        lordba.gated_backward(h, h, h, dgate=h, dup=torch.zeros_like(h))          # dgate over dh
    with pytest.raises(lordba.LordbaError):
        lordba.dropout(x, 1.5, 0)
    with pytest.raises(lordba.LordbaError):
        lordba.dropout(x[:, :32], 0.5, 0, out=x[:, 16:48])                       # overlapping, not the same
    clean()


@pytest.mark.parametrize("tokens,d_model,d_hidden", [(3, 128, 320), (150, 256, 700)])
def test_the_adapted_block_of_the_example(tokens, d_model, d_hidden):
    """Served and trained against the same block in float32.  A dozen bfloat16 roundings (2^-9 each in the mean)
    lie between the two; in the served path a value near a step of the 8-bit grid may land on the other side
    (1/127 of a row's largest entry, for the few entries that do)."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "adapted_feed_forward.py")
    spec = importlib.util.spec_from_file_location("adapted_feed_forward", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    errors = example.run(tokens, d_model, d_hidden, 8)
    assert set(errors) == {"served", "output", "dx", "dw_gate", "dw_up"}
    assert all(e < 12 * 2.0 ** -9 for e in errors.values()), errors
