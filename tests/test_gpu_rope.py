"""GPU parity of the norms of queries and keys with the rotation, and of their gradients, against float64 implementations
written here.

Tolerances, from the arithmetic (u as in test_gpu_block): the mean of d squares, its root and the products after it are
good to (d + 8) 2^-24; cosine and sine to 2^-21 (the angle's last whole turn taken off, 2^-24 of a turn is left, and the
functions' own two units); a rotated entry is a sum of two such products.  E = (d + 64) 2^-23 covers both with room for
the order of sums.  A sum over n head vectors may lose another n 2^-24 of its magnitudes.
"""
import math

import numpy as np
import pytest
import torch

from paper_2605_24058_b200 import lordba
from test_gpu_block import TINY, TYPES, UNIT, f64

pytestmark = pytest.mark.gpu


def heads(rng, T, H, d, dtype, pad=0, lead=0, scale=1.5):
    """(device view, float64 values): heads side by side, pad entries behind a token's last, lead before the first."""
    buf = torch.from_numpy((rng.standard_normal(T * (H * d + pad) + lead) * scale).astype(np.float32)).to(TYPES[dtype]).cuda()
    t = buf[lead:].view(T, H * d + pad)[:, :H * d].unflatten(1, (H, d))
    return t, f64(t)


def turn(v, positions, inv_freq, interleaved, back=False):
    """v rotated, and the sum of magnitudes that makes up an entry."""
    R = 2 * len(inv_freq)
    angle = positions.astype(np.float64)[:, None] * inv_freq.astype(np.float64)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None] * (-1 if back else 1)
    a, b = (np.arange(0, R, 2), np.arange(1, R, 2)) if interleaved else (np.arange(R // 2), np.arange(R // 2, R))
    out, size = v.copy(), np.abs(v)
    out[..., a], out[..., b] = v[..., a] * c - v[..., b] * s, v[..., b] * c + v[..., a] * s
    size[..., a] = size[..., b] = np.abs(v[..., a]) + np.abs(v[..., b])
    return out, size


def check(got, want, bound, dtype, what):
    got = f64(got)
    tol = bound + UNIT[dtype] * (np.abs(want) + bound) + TINY[dtype]
    bad = ~(np.abs(got - want) <= tol)
    assert got.shape == want.shape and not bad.any(), "%s: %d of %d off, first at %s: got %r want %r tol %r" % (
        what, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0], tol[bad][0])


def forward(v, w, positions, inv_freq, eps, norm, interleaved):
    if norm:
        v = v / np.sqrt((v * v).mean(-1, keepdims=True) + eps) * w
    return turn(v, positions, inv_freq, interleaved)


def backward(g, v, w, positions, inv_freq, eps, norm, interleaved):
    """(dx, its magnitudes, dw, its magnitudes)"""
    g, size = turn(g, positions, inv_freq, interleaved, back=True)
    if not norm:
        return g, size, None, None
    r = 1 / np.sqrt((v * v).mean(-1, keepdims=True) + eps)
    x = v * r
    dx = r * (g * w - x * (g * w * x).mean(-1, keepdims=True))
    big = r * (size * np.abs(w) + np.abs(x) * (size * np.abs(w * x)).mean(-1, keepdims=True))
    return dx, big, (g * x).sum((0, 1)), (size * np.abs(x)).sum((0, 1))


def frequencies(R):
    return (10000.0 ** (-np.arange(0, R, 2) / max(R, 1))).astype(np.float32)


SHAPES = [  # T, heads_q, heads_k, d, rotary, interleaved, pad, lead
    (1, 1, 1, 2, 2, False, 0, 0), (1, 32, 32, 128, 128, False, 0, 0), (1, 5, 0, 64, 64, True, 0, 0), (3, 4, 1, 1, 0, False, 0, 0), (2, 3, 2, 7, 4, False, 0, 0),
    (7, 8, 2, 128, 128, False, 0, 0), (9, 6, 3, 64, 32, False, 8, 0), (17, 2, 2, 80, 80, True, 0, 0), (33, 5, 1, 80, 40, False, 0, 0), (65, 4, 4, 96, 96, False, 5, 1),
    (40, 3, 1, 512, 512, False, 0, 0), (12, 2, 1, 511, 510, True, 0, 0), (21, 4, 2, 256, 64, True, 64, 0), (200, 16, 4, 128, 128, False, 1024, 8), (500, 32, 8, 64, 64, False, 0, 0),
    (300, 1, 1, 24, 16, False, 0, 0), (130, 2, 1, 33, 32, False, 3, 0), (1000, 7, 3, 128, 64, True, 0, 0), (50, 40, 40, 16, 16, False, 0, 0), (19, 2, 2, 72, 48, False, 0, 0),
    (77, 4, 2, 128, 128, False, 5, 1), (30, 2, 1, 64, 64, True, 3, 0), (26, 3, 2, 256, 256, False, 1, 7), (44, 5, 2, 128, 64, False, 5, 3), (31, 2, 2, 80, 80, True, 7, 0)]


@pytest.mark.parametrize("T,hq,hk,d,R,interleaved,pad,lead", SHAPES)
@pytest.mark.parametrize("dtype,norm,wtype", [("bf16", True, "bf16"), ("f16", False, None), ("f32", True, "f32"), ("f16", True, None)])
def test_norm_rope(T, hq, hk, d, R, interleaved, pad, lead, dtype, norm, wtype):
    rng = np.random.default_rng(T * 7 + d)
    inv = frequencies(R)
    pos = rng.integers(-5, 200000, T)
    q, vq = heads(rng, T, hq, d, dtype, pad, lead)
    k, vk = heads(rng, T, max(hk, 1), d, dtype, pad, lead)
    weights = [torch.from_numpy((1 + 0.3 * rng.standard_normal(d)).astype(np.float32)).to(TYPES[wtype]).cuda() if wtype else None for _ in range(2)]
    values = [f64(w) if w is not None else np.ones(d) for w in weights]
    args = (torch.from_numpy(pos).cuda(), torch.from_numpy(inv).cuda(), weights[0], weights[1] if hk else None)
    kw = dict(eps=1e-5, norm=norm, interleaved=interleaved)
    E = (d + 64) * 2.0 ** -23
    keys = k if hk else None
    got = lordba.norm_rope(q, keys, *args, **kw)
    assert (got[1] is None) == (hk == 0)
    sides = [(0, vq, hq)] + ([(1, vk, hk)] if hk else [])
    for i, v, h in sides:
        want, size = forward(v, values[i], pos, inv, np.float32(1e-5), norm, interleaved)
        check(got[i], want, E * size, dtype, "qk"[i])
    # outputs of the caller's with room between heads, and in place: another layout may add its squares in another order, which
    # the bound allows for
    wants = [forward(v, values[i], pos, inv, np.float32(1e-5), norm, interleaved) for i, v, h in sides]
    room = torch.full((T, hq, d + 3), 77.0, dtype=TYPES[dtype], device="cuda")
    lordba.norm_rope(q, keys, *args, q_out=room[..., :d], **kw)
    check(room[..., :d], wants[0][0], E * wants[0][1], dtype, "q with room")
    assert (room[..., d:] == 77).all()
    q2, k2 = q.clone(), keys.clone() if hk else None
    lordba.norm_rope(q2, k2, *args, q_out=q2, k_out=k2, **kw)
    for i, t in enumerate((q2, k2)[:len(sides)]):
        check(t, wants[i][0], E * wants[i][1], dtype, "in place")


@pytest.mark.parametrize("T,hq,hk,d,R,interleaved,pad,lead", SHAPES)
@pytest.mark.parametrize("dtype,norm,wtype", [("bf16", True, "f32"), ("f16", False, None), ("f32", True, "f32"), ("bf16", True, None)])
def test_norm_rope_backward(T, hq, hk, d, R, interleaved, pad, lead, dtype, norm, wtype):
    rng = np.random.default_rng(T * 11 + d)
    inv = frequencies(R)
    pos = rng.integers(-5, 200000, T)
    n = max(hk, 1)
    q, vq = heads(rng, T, hq, d, dtype, pad, lead)
    k, vk = heads(rng, T, n, d, dtype, 0, 0)
    gq, vgq = heads(rng, T, hq, d, dtype, pad, lead, 1.0)
    gk, vgk = heads(rng, T, n, d, dtype, 0, 0, 1.0)
    weights = [torch.from_numpy((1 + 0.3 * rng.standard_normal(d)).astype(np.float32)).to(TYPES[wtype]).cuda() if wtype else None for _ in range(2)]
    values = [f64(w) if w is not None else np.ones(d) for w in weights]
    args = (torch.from_numpy(pos).cuda(), torch.from_numpy(inv).cuda(), weights[0], weights[1] if hk else None)
    kw = dict(eps=1e-5, norm=norm, interleaved=interleaved)
    keys, dkeys = (k, gk) if hk else (None, None)
    got = lordba.norm_rope_backward(gq, dkeys, q, keys, *args, **kw)
    E = (d + 64) * 2.0 ** -22
    sides = [(0, vgq, vq, hq)] + ([(1, vgk, vk, hk)] if hk else [])
    for i, g, v, h in sides:
        dx, big, dw, dbig = backward(g, v, values[i], pos, inv, np.float32(1e-5), norm, interleaved)
        check(got[i], dx, E * big, dtype, "d" + "qk"[i])
        assert (got[2 + i] is not None) == (wtype is not None)
        if wtype:
            check(got[2 + i], dw, (E + T * h * 2.0 ** -24) * dbig, "f32", "dw")
    assert hk or (got[1] is None and got[3] is None)
    # over the gradient's own place
    gq2 = gq.clone()
    again = lordba.norm_rope_backward(gq2, dkeys, q, keys, *args, dq=gq2, **kw)
    dx, big, dw, dbig = backward(vgq, vq, values[0], pos, inv, np.float32(1e-5), norm, interleaved)
    check(again[0], dx, E * big, dtype, "dq in place")
    if wtype:
        check(again[2], dw, (E + T * hq * 2.0 ** -24) * dbig, "f32", "dw")


def test_gradients_are_differences():
    """The derivative along a direction, of a weighted sum of the results in float32: central differences of step h are off by
    h^2 / 6 of a third derivative (below 60 |v|^3 here, head vectors are about 1) and by the rounding of two results."""
    rng = np.random.default_rng(5)
    T, H, d = 4, 2, 32
    q, vq = heads(rng, T, H, d, "f32", scale=1.0)
    c, vc = heads(rng, T, H, d, "f32", scale=1.0)
    v, vv = heads(rng, T, H, d, "f32", scale=1.0)
    w = torch.from_numpy(rng.standard_normal(d).astype(np.float32)).cuda()
    dw_dir = torch.from_numpy(rng.standard_normal(d).astype(np.float32)).cuda()
    pos, inv = torch.tensor([0, 3, 70, 1000]).cuda(), torch.from_numpy(frequencies(d)).cuda()
    f = lambda x, w: float((lordba.norm_rope(x, None, pos, inv, w)[0].double() * c.double()).sum())
    dq, _, dw, _ = lordba.norm_rope_backward(c, None, q, None, pos, inv, w)
    h = 2.0 ** -8
    size = float((np.abs(vc)).sum() * 8)
    tol = h * h / 6 * 60 * float((np.abs(vv) ** 3).sum()) + 2 * size * 2.0 ** -22 / h
    along = (f(q + h * v, w) - f(q - h * v, w)) / (2 * h)
    assert abs(along - float((dq.double() * v.double()).sum())) <= tol
    along = (f(q, w + h * dw_dir) - f(q, w - h * dw_dir)) / (2 * h)               # linear in w: rounding alone
    assert abs(along - float((dw.double() * dw_dir.double()).sum())) <= 2 * size * 2.0 ** -22 / h


def test_far_positions_and_other_layouts():
    """Positions beyond 32 bits, heads before tokens, one head that all share, tensors longer than 32 bits count."""
    rng = np.random.default_rng(1)
    T, H, d = 6, 4, 64
    inv = frequencies(d)
    pos = np.array([0, 1 << 20, (1 << 31) - 1, (1 << 31) + 5, -(1 << 31), 1 << 33])
    by_head = torch.from_numpy(rng.standard_normal((H, T, d)).astype(np.float32)).cuda()
    q = by_head.transpose(0, 1)
    one = by_head[:1].transpose(0, 1).expand(T, 3, d)
    out, k_out = lordba.norm_rope(q, one, torch.from_numpy(pos).cuda(), torch.from_numpy(inv).cuda())
    for got, v in ((out, f64(q)), (k_out, f64(one))):
        want, size = forward(v, 1.0, pos, inv, np.float32(1e-6), True, False)
        # 2^33 radians in 64 bits are good to 2^-19
        check(got, want, (2.0 ** -18 + (d + 64) * 2.0 ** -23) * size, "f32", "far")
    q_out = torch.empty_like(by_head).transpose(0, 1)
    lordba.norm_rope(q, None, torch.from_numpy(pos).cuda(), torch.from_numpy(inv).cuda(), q_out=q_out)
    assert torch.equal(q_out, out)              # both aligned: the same way
    far = (1 << 30) + 8
    big = torch.zeros(2 * far + H * d, dtype=torch.bfloat16, device="cuda")
    view = big.as_strided((3, H, d), (far, d, 1))
    small = torch.randn(3, H, d, device="cuda").to(torch.bfloat16)
    view.copy_(small)
    where = torch.arange(3, device="cuda")
    want = lordba.norm_rope(small, None, where, torch.from_numpy(inv).cuda())[0]
    lordba.norm_rope(view, None, where, torch.from_numpy(inv).cuda(), q_out=view)
    assert torch.equal(view, want)


def test_rows_of_zeros_and_numbers_that_are_not_finite():
    T, H, d, R = 5, 3, 64, 32
    x = torch.randn(T, H, d, device="cuda")
    x[1, 1] = 0
    x[2, 0, 40] = math.inf                # behind the rotated entries
    x[3, 2, 3] = math.nan
    pos, inv = torch.arange(T, device="cuda"), torch.from_numpy(frequencies(R)).cuda()
    y = lordba.norm_rope(x, None, pos, inv)[0]
    bad = ~torch.isfinite(y).all(-1)
    assert bad.sum() == 2 and bad[2, 0] and bad[3, 2] and (y[1, 1] == 0).all()
    y = lordba.norm_rope(x, None, pos, inv, norm=False)[0]
    assert y[2, 0, 40] == math.inf and torch.isfinite(y[2, 0, :40]).all() and torch.isnan(y[3, 2]).sum() == 2 and torch.equal(y[..., R:], x[..., R:])


def test_streams_graphs_and_no_tokens():
    rng = np.random.default_rng(9)
    T, d = 300, 128
    q, _ = heads(rng, T, 8, d, "bf16")
    k, _ = heads(rng, T, 2, d, "bf16")
    w = torch.rand(d, device="cuda")
    pos, inv = torch.arange(T, device="cuda"), torch.from_numpy(frequencies(d)).cuda()
    want = lordba.norm_rope_backward(q, k, q, k, pos, inv, w, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = lordba.norm_rope_backward(q, k, q, k, pos, inv, w, w, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ws = torch.empty(8 << 20, dtype=torch.uint8, device="cuda")
    outs = [torch.zeros_like(t) for t in want]
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            lordba.norm_rope_backward(q, k, q, k, pos, inv, w, w, dq=outs[0], dk=outs[1], dw_q=outs[2], dw_k=outs[3], workspace=ws)
    for g in graphs * 2:
        for t in outs:
            t.zero_()
        g.replay()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    none = lordba.norm_rope_backward(q[:0], k[:0], q[:0], k[:0], pos[:0], inv, w, w)
    assert none[0].shape == (0, 8, d) and (none[2] == 0).all() and (none[3] == 0).all()
    assert lordba.norm_rope(q[:0], None, pos[:0], inv)[0].shape == (0, 8, d)


def test_refusals():
    rng = np.random.default_rng(0)
    q, _ = heads(rng, 4, 2, 64, "bf16")
    pos, inv = torch.arange(4, device="cuda"), torch.ones(32, device="cuda")
    w = torch.ones(64, device="cuda")
    call = lambda q=q, k=None, pos=pos, inv=inv, w_q=None, w_k=None, **kw: lordba.norm_rope(q, k, pos, inv, w_q, w_k, **kw)
    assert call()[0].shape == q.shape
    for wrong, error in [(dict(q=q[0]), ValueError), (dict(q=q.transpose(1, 2)), ValueError), (dict(pos=pos.int()), TypeError), (dict(pos=pos[:3]), TypeError),
                         (dict(inv=inv.double()), TypeError), (dict(inv=torch.ones(33, device="cuda")), ValueError), (dict(w_q=w[:63]), ValueError),
                         (dict(w_k=w), ValueError), (dict(k=q.float()), TypeError), (dict(k=q[:3]), ValueError), (dict(k_out=q), ValueError),
                         (dict(q=q.cpu()), ValueError), (dict(q=q.int()), TypeError), (dict(q_out=q.float()), TypeError), (dict(w_q=w, k=q, w_k=w.half()), TypeError)]:
        with pytest.raises(error):
            call(**wrong)
    for wrong in (dict(eps=-1.0), dict(w_q=w, norm=False), dict(q_out=q[:1].expand(4, 2, 64)), dict(q=q[:, :1].expand(4, 2, 64), q_out=q)):
        with pytest.raises(lordba.LordbaError):
            call(**wrong)
    with pytest.raises(RuntimeError, match="gradient"):
        call(w_q=w.clone().requires_grad_(True))
    with pytest.raises(lordba.LordbaError):
        lordba.norm_rope_backward(q, None, q, None, pos, inv, w, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
