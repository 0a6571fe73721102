"""GPU parity of the products with 4-bit weights and group scales against plain float64 implementations written here.

Tolerances, from the arithmetic; u is the unit roundoff of the type (bf16 2^-8, f16 2^-11; f16 results below 2^-14 are
multiples of 2^-24).
  carrier: integers are exact, and so is the weight scale * (u - zero) before its one rounding.
  products: each of the K additions of a float32 sum may lose 2^-23 of the sum of magnitudes (truncating adders); where
    the weights enter in 16 bits each is off by u of itself (a weight below 2^-14 in f16 by 2^-25); the result is
    rounded once more.
"""
import math

import numpy as np
import pytest
import torch

from paper_2605_24058_b200 import lordba
from test_gpu_block import TINY, TYPES, UNIT, clean, close, f64, matrix, target, untouched

pytestmark = pytest.mark.gpu


def carrier_bytes(u):
    """The carrier of 4-bit values (d_out, d_in), by the layout that the header states."""
    n, d = u.shape
    out = np.zeros((n, lordba.int4_row_bytes(d) // 4), dtype=np.uint32)
    for k in range(d):
        block, col = divmod(k, 128)
        j, rest = divmod(col, 32)
        t, c = divmod(rest, 8)
        out[:, 16 * block + 4 * t + j] |= u[:, k].astype(np.uint32) << np.uint32(4 * (c // 2) + 16 * (c % 2))
    return out.view(np.uint8)


class Weights:
    """A random matrix of 4-bit weights: what the calls take, and its float64 values.  The carrier, scales and zeros are
    parts of larger tensors, full of other things, where padded."""

    def __init__(self, rng, n, d, group, zeros, dtype, padded=False, gain=1.0):
        g = -(-d // group)
        self.u = rng.integers(0, 16, (n, d), dtype=np.uint8)
        self.q = lordba.int4_pack(torch.from_numpy(self.u).cuda())
        scale = torch.from_numpy(np.exp(rng.standard_normal((n, g)) * 0.5).astype(np.float32) * np.float32(gain / math.sqrt(8 * d))).to(TYPES[dtype]).cuda()
        zero = torch.from_numpy(rng.integers(0, 16, (n, g), dtype=np.uint8)).cuda() if zeros else None
        self.group = group
        spread = lambda v: np.repeat(v, group, axis=1)[:, :d]
        self.v = spread(f64(scale)) * (self.u - (spread(zero.cpu().numpy()).astype(np.float64) if zeros else 8.0))
        if padded:
            def inside(t, rows, cols, fill):
                big = torch.full((t.shape[0] + rows, t.shape[1] + cols), fill, dtype=t.dtype, device="cuda")
                big[rows:, :t.shape[1]] = t
                return big[rows:, :t.shape[1]]
            self.q, scale = inside(self.q, 3, 48, 255), inside(scale, 1, 3, math.nan)
            zero = inside(zero, 1, 5, 255) if zeros else None
        self.scale, self.zero = scale, zero

    def args(self):
        return dict(zero=self.zero, group=self.group)


def product_bound(a, b, dtype):
    """|err| of a @ b before the last rounding, b the weights."""
    K = a.shape[1]
    return (K * 2.0 ** -23 + UNIT[dtype]) * (np.abs(a) @ np.abs(b)) + TINY[dtype] * np.abs(a).sum(1, keepdims=True)


# ------------------------------------------------------------------------------------------------ the carrier

@pytest.mark.parametrize("n,d", [(1, 1), (3, 7), (5, 128), (2, 129), (70000, 33), (9, 1000), (4, 4096)])
def test_pack_lays_out_what_the_header_says(n, d):
    u = np.random.default_rng(d).integers(0, 256, (n, d), dtype=np.uint8)
    q = lordba.int4_pack(torch.from_numpy(u).cuda())
    assert q.shape == (n, lordba.int4_row_bytes(d)) and np.array_equal(q.cpu().numpy(), carrier_bytes(u & 15))
    buf = torch.full((n, q.shape[1] + 16), 99, dtype=torch.uint8, device="cuda")
    assert lordba.int4_pack(torch.from_numpy(np.pad(u, ((0, 0), (0, 3)))).cuda()[:, :d], q=buf[:, :q.shape[1]]) is not None
    assert torch.equal(buf[:, :q.shape[1]], q) and (buf[:, q.shape[1]:] == 99).all()


@pytest.mark.parametrize("n,d,group", [(1, 1, 32), (3, 7, 32), (16, 256, 32), (5, 129, 64), (33, 1000, 128), (7, 300, 512), (2, 11008, 16384), (300, 64, 32)])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_dequantize(n, d, group, zeros, dtype):
    w = Weights(np.random.default_rng(n * 3 + d), n, d, group, zeros, dtype, padded=True)
    want = torch.from_numpy(w.v).to(TYPES[dtype])                     # the one rounding
    assert torch.equal(lordba.int4_dequantize(w.q, w.scale, d, **w.args()).cpu(), want)
    buf, out = target(n, d, dtype, 5, 1)
    lordba.int4_dequantize(w.q, w.scale, d, w=out, **w.args())
    assert torch.equal(out.cpu(), want)
    untouched(buf, n, d, 5, 1)


def nearest(w, s):
    """w / s to whole numbers, ties to even: the quotient of numbers of at most 24 bits is never so close to a half that
    float64 could not tell."""
    return np.rint(w / np.where(s > 0, s, 1.0))


@pytest.mark.parametrize("n,d,group,pad", [(1, 1, 32, 0), (3, 7, 32, 2), (70000, 40, 32, 0), (64, 256, 64, 0), (33, 1000, 128, 3), (9, 3000, 1024, 0), (4, 777, 65536, 0)])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("wtype,dtype", [("f32", "f16"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16")])
def test_quantize(n, d, group, pad, zeros, wtype, dtype):
    rng = np.random.default_rng(n + d)
    w, v = matrix(rng, n, d, wtype, pad, 0.02)
    q, scale, zero = lordba.int4_quantize(w, group, zeros, dtype=TYPES[dtype])
    assert scale.dtype == TYPES[dtype] and (zero is not None) == zeros
    g = -(-d // group)
    wide = np.pad(v, ((0, 0), (0, g * group - d))).reshape(n, g, group).astype(np.float32)
    low, high = np.minimum(wide.min(2), 0), np.maximum(wide.max(2), 0)
    s32 = (high - low) / np.float32(15) if zeros else np.maximum(high, -low) / np.float32(7)
    s = f64(torch.from_numpy(s32).to(TYPES[dtype]))
    assert np.array_equal(f64(scale), s)
    z = np.where(s > 0, np.minimum(nearest(-low.astype(np.float64), s), 15), 8) if zeros else np.full((n, g), 8.0)
    if zeros:
        assert np.array_equal(zero.cpu().numpy(), z)
    u = np.where(s[..., None] > 0, np.clip(nearest(wide.astype(np.float64), s[..., None]) + z[..., None], 0, 15), 8)
    u = u.reshape(n, g * group)[:, :d]
    blocks = lordba.int4_row_bytes(d) * 2
    want = carrier_bytes(np.pad(u, ((0, 0), (0, blocks - d))).astype(np.uint8))
    got = q.cpu().numpy()
    inside = carrier_bytes(np.pad(np.full((1, d), 15, np.uint8), ((0, 0), (0, blocks - d))))
    assert np.array_equal(got & inside, want & inside)


def test_quantize_groups_without_a_scale():
    w = torch.randn(8, 256, device="cuda")
    w[1, 64:128] = 0
    w[2, 70] = math.inf
    w[3, 200] = math.nan
    w[4, :64] *= 1e-12                    # the scale rounds to zero in float16
    w[5, 0] = -1e30                       # and here it overflows
    for zeros in (False, True):
        q, scale, zero = lordba.int4_quantize(w, 64, zeros, dtype=torch.float16)
        s = scale.float().cpu().numpy()
        bad = np.isnan(s)
        assert bad.sum() == 3 and bad[2, 1] and bad[3, 3] and bad[5, 0] and s[1, 1] == 0 and s[4, 0] == 0
        x = torch.ones(3, 256, dtype=torch.float16, device="cuda")
        y = lordba.int4_linear(x, q, scale, zero, 64).float().cpu().numpy()
        assert np.isnan(y[:, [2, 3, 5]]).all() and np.isfinite(y[:, [0, 1, 4, 6, 7]]).all()
        back = lordba.int4_dequantize(q, scale, 256, zero, 64).float().cpu().numpy()
        assert (back[1, 64:128] == 0).all() and (back[4, :64] == 0).all() and np.isnan(back[2, 64:128]).all() and np.isfinite(back[2, 128:]).all()


def test_quantize_halves_go_to_even():
    """Quotients of exactly a half, and one step to either side of it."""
    s = 2.0 ** -6
    k = np.arange(-6, 7) + 0.5
    w = np.concatenate([k * s, np.nextafter(np.float32(k * s), np.float32(9)), np.nextafter(np.float32(k * s), np.float32(-9)), [7 * s]]).astype(np.float32)
    q, scale, _ = lordba.int4_quantize(torch.from_numpy(w[None]).cuda(), 64, dtype=torch.float16)
    assert float(scale[0, 0]) == s
    back = lordba.int4_dequantize(q, scale, w.size, group=64).float().cpu().numpy()[0] / s
    assert np.array_equal(back, np.rint(w.astype(np.float64) / s))


# ------------------------------------------------------------------------------------------------ the product

SIZES = [  # T, d_in, d_out, group, pad, lead
    (1, 1, 1, 32, 0, 0), (1, 4096, 1000, 128, 0, 0), (1, 130, 17, 32, 0, 0), (1, 11008, 64, 64, 0, 0), (1, 96, 5000, 32, 0, 1), (2, 128, 128, 128, 0, 0),
    (3, 1001, 131, 32, 5, 1), (4, 8192, 40, 16384, 0, 0), (5, 2048, 640, 256, 0, 0), (8, 2048, 129, 64, 8, 0), (9, 512, 300, 32, 0, 0), (15, 777, 33, 64, 3, 0),
    (16, 4096, 256, 128, 0, 0), (17, 640, 257, 32, 0, 0), (31, 129, 96, 64, 16, 0), (32, 1024, 200, 128, 0, 0), (33, 256, 1000, 64, 1, 3), (56, 4096, 384, 128, 0, 0),
    (64, 1111, 333, 32, 0, 0), (65, 640, 512, 128, 0, 0), (128, 2048, 260, 64, 0, 0), (129, 160, 1025, 32, 0, 0), (200, 3000, 136, 128, 8, 0), (256, 512, 256, 128, 0, 0),
    (300, 1001, 700, 64, 7, 1), (513, 384, 520, 128, 0, 0), (777, 96, 1533, 32, 0, 0), (1100, 320, 600, 128, 5, 0)]


@pytest.mark.parametrize("T,d_in,d_out,group,pad,lead", SIZES)
@pytest.mark.parametrize("dtype,zeros", [("bf16", False), ("f16", True)])
def test_int4_linear(T, d_in, d_out, group, pad, lead, dtype, zeros):
    rng = np.random.default_rng(T * 31 + d_in)
    x, vx = matrix(rng, T, d_in, dtype, pad, 1.0, lead)
    w = Weights(rng, d_out, d_in, group, zeros, dtype, padded=pad > 0)
    buf, y = target(T, d_out, dtype, pad, lead)
    assert lordba.int4_linear(x, w.q, w.scale, y=y, **w.args()) is y
    clean()
    close(y, vx @ w.v.T, product_bound(vx, w.v.T, dtype), dtype, "y")
    untouched(buf, T, d_out, pad, lead)


@pytest.mark.parametrize("T,d_in,d_out,group,pad,lead", SIZES)
@pytest.mark.parametrize("dtype,zeros", [("bf16", True), ("f16", False)])
def test_int4_linear_backward(T, d_in, d_out, group, pad, lead, dtype, zeros):
    rng = np.random.default_rng(T * 37 + d_out)
    dy, vy = matrix(rng, T, d_out, dtype, pad, 1.0, lead)
    w = Weights(rng, d_out, d_in, group, zeros, dtype, padded=pad > 0)
    buf, dx = target(T, d_in, dtype, pad, lead)
    assert lordba.int4_linear_backward(dy, w.q, w.scale, d_in, dx=dx, **w.args()) is dx
    clean()
    close(dx, vy @ w.v, product_bound(vy, w.v, dtype), dtype, "dx")
    untouched(buf, T, d_in, pad, lead)


@pytest.mark.parametrize("T", [1, 8, 40, 300])
def test_what_lies_outside_is_not_looked_at(T):
    """Columns of x behind the last one, and of the carrier: NaN in the one, anything in the other."""
    rng = np.random.default_rng(T)
    d_in, d_out = 200, 150
    w = Weights(rng, d_out, d_in, 32, True, "bf16")
    x = torch.full((T, 256), math.nan, dtype=torch.bfloat16, device="cuda")
    x[:, :d_in] = torch.from_numpy(rng.standard_normal((T, d_in)).astype(np.float32))
    first = lordba.int4_linear(x[:, :d_in], w.q, w.scale, **w.args())
    assert torch.isfinite(first).all()
    rest = torch.from_numpy(carrier_bytes(np.pad(np.zeros((1, d_in), np.uint8), ((0, 0), (0, 56)), constant_values=15))).cuda()
    q = w.q | rest
    assert not torch.equal(q, w.q)
    assert torch.equal(lordba.int4_linear(x[:, :d_in], q, w.scale, **w.args()), first)
    dy = torch.from_numpy(rng.standard_normal((T, d_out)).astype(np.float32)).to(torch.bfloat16).cuda()
    assert torch.equal(lordba.int4_linear_backward(dy, q, w.scale, d_in, **w.args()), lordba.int4_linear_backward(dy, w.q, w.scale, d_in, **w.args()))


@pytest.mark.parametrize("T", [1, 7, 40, 300])
def test_numbers_that_are_not_finite_stay_in_their_row(T):
    rng = np.random.default_rng(T)
    w = Weights(rng, 140, 256, 64, False, "bf16")
    x, _ = matrix(rng, T, 256, "bf16")
    dy, _ = matrix(rng, T, 140, "bf16")
    w.scale[5, 2], w.scale[7, 0] = math.nan, math.inf
    y = lordba.int4_linear(x, w.q, w.scale, group=64).float()
    rows = torch.arange(140, device="cuda")
    assert not torch.isfinite(y[:, [5, 7]]).any() and torch.isfinite(y[:, (rows != 5) & (rows != 7)]).all()
    dx = lordba.int4_linear_backward(dy, w.q, w.scale, 256, group=64).float()
    assert torch.isnan(dx[:, 128:192]).all() and not torch.isfinite(dx[:, :64]).all() and torch.isfinite(dx[:, 64:128]).all() and torch.isfinite(dx[:, 192:]).all()
    w = Weights(rng, 140, 256, 64, False, "bf16")
    x[T - 1, 9] = math.inf
    y = lordba.int4_linear(x, w.q, w.scale, group=64).float()
    assert torch.isfinite(y[:T - 1]).all() and not torch.isfinite(y[T - 1]).any()


def test_a_zero_point_has_four_bits():
    rng = np.random.default_rng(3)
    w = Weights(rng, 64, 256, 64, True, "f16")
    for T in (2, 300):
        x, _ = matrix(rng, T, 256, "f16")
        want = lordba.int4_linear(x, w.q, w.scale, w.zero, 64)
        assert torch.equal(lordba.int4_linear(x, w.q, w.scale, w.zero + 240, 64), want)


@pytest.mark.parametrize("T", [1, 16, 48, 400])
def test_streams_graphs_and_repeats(T):
    """The same bits from run to run, on another stream, from two graphs that share a workspace."""
    rng = np.random.default_rng(T)
    w = Weights(rng, 520, 1024, 128, True, "bf16")
    x, _ = matrix(rng, T, 1024, "bf16")
    dy, _ = matrix(rng, T, 520, "bf16")
    forward = lambda **kw: lordba.int4_linear(x, w.q, w.scale, w.zero, 128, **kw)
    backward = lambda **kw: lordba.int4_linear_backward(dy, w.q, w.scale, 1024, w.zero, 128, **kw)
    want = forward(), backward()
    for _ in range(5):
        assert torch.equal(forward(), want[0]) and torch.equal(backward(), want[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = forward(stream=side), backward(stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    y, dx = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    with torch.cuda.stream(side):
        forward(y=y, workspace=ws)
        backward(dx=dx, workspace=ws)
    side.synchronize()
    one, two = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(one):
        forward(y=y, workspace=ws)
    with torch.cuda.graph(two):
        backward(dx=dx, workspace=ws)
    for _ in range(3):
        y.zero_()
        dx.zero_()
        one.replay()
        two.replay()
        assert torch.equal(y, want[0]) and torch.equal(dx, want[1])
    clean()


def test_refusals():
    rng = np.random.default_rng(0)
    w = Weights(rng, 64, 256, 64, True, "bf16")
    x, _ = matrix(rng, 4, 256, "bf16")
    call = lambda x=x, q=w.q, scale=w.scale, zero=w.zero, group=64, **kw: lordba.int4_linear(x, q, scale, zero, group, **kw)
    assert call().shape == (4, 64)
    for wrong, error in [(dict(x=x.float()), TypeError), (dict(x=x.half()), TypeError), (dict(scale=w.scale.float()), TypeError), (dict(zero=w.zero.int()), TypeError),
                         (dict(group=48), ValueError), (dict(group=0), ValueError), (dict(group=128), ValueError), (dict(x=x[0]), ValueError),
                         (dict(x=x.t()), ValueError), (dict(q=w.q[:63]), ValueError), (dict(q=w.q[:, :64]), ValueError), (dict(x=x.cpu()), ValueError),
                         (dict(scale=w.scale[:, :2]), ValueError), (dict(y=torch.empty(4, 63, dtype=x.dtype, device="cuda")), ValueError), (dict(q=None), TypeError)]:
        with pytest.raises(error):
            call(**wrong)
    with pytest.raises(lordba.LordbaError, match="unsupported"):
        lordba.int4_linear(x.float(), w.q, w.scale.float(), w.zero, 64)
    with pytest.raises(RuntimeError, match="gradient"):
        call(x=x.clone().requires_grad_(True))
    with pytest.raises(lordba.LordbaError):
        call(y=torch.as_strided(x, (4, 64), (256, 1)))                      # y inside x
    with pytest.raises(ValueError):
        lordba.int4_linear_backward(x[:, :64], w.q, w.scale, 0, w.zero, 64)
    big = Weights(rng, 64, 256, 64, False, "bf16")
    with pytest.raises(lordba.LordbaError):
        lordba.int4_linear(matrix(rng, 300, 256, "bf16")[0], big.q, big.scale, group=64, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert call(x=x[:0]).shape == (0, 64)


@pytest.mark.parametrize("T", [1, 3])
def test_rows_of_more_than_two_gigabytes(T):
    """Columns whose byte offsets pass 31 bits; nearly all of x is zero, so that the sums are exact."""
    d_in, d_out, group = (1 << 30) + 200, 2, 1 << 16
    x = torch.zeros(T, d_in + 56, dtype=torch.float16, device="cuda")
    q = torch.randint(0, 256, (d_out, lordba.int4_row_bytes(d_in)), dtype=torch.uint8, device="cuda")
    scale = torch.full((d_out, -(-d_in // group)), 0.25, dtype=torch.float16, device="cuda")
    at = [0, 5, 127, 128, (1 << 29) + 3, (1 << 30) - 1, 1 << 30, d_in - 1]
    want = np.zeros((T, d_out))
    host = {}
    for c in at:
        block, col = divmod(c, 128)
        j, rest = divmod(col, 32)
        t, e = divmod(rest, 8)
        words = q[:, 64 * block + 4 * (4 * t + j):64 * block + 4 * (4 * t + j) + 4].cpu().numpy().copy().view(np.uint32)[:, 0]
        host[c] = (words >> np.uint32(4 * (e // 2) + 16 * (e % 2))) & 15
    for i, c in enumerate(at):
        for token in {0, T - 1}:
            x[token, c] = i + 1 + token
            want[token] += (i + 1 + token) * 0.25 * (host[c].astype(np.float64) - 8)
    x[:, d_in:] = math.nan
    y = lordba.int4_linear(x[:, :d_in], q, scale, None, group)
    assert np.array_equal(f64(y), want)
    clean()
