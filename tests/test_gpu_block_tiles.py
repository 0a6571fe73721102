"""The tile kernel over several tiles a CTA pair: accumulators, rings and the epilogue's patches are used again, the
last columns are fewer than the copy engine writes at a time, and some outputs are within its reach while others
are not.  Results are held to float64 products formed on the device, every call is made several times (an
epilogue that overtakes its own stores would not give the same bits), and nothing beside the rows is touched.

Tolerances as in test_gpu_block.py: K 2^-23 sum |a b| of a float32 sum of K products (4 float32 roundings of an
8-bit one), 2^-18 of the activation, the slope of the activation at most 1.13, then the output's rounding."""
import math

import pytest
import torch

from paper_2605_24058_b200 import lordba
from test_gpu_block import TINY, TYPES, UNIT

pytestmark = pytest.mark.gpu


def draws(gen, rows, cols, dtype, scale=1.0, pad=0):
    buf = torch.randn(rows, cols + pad, generator=gen, device="cuda").mul_(scale)
    return buf.to(TYPES[dtype])[:, :cols]


def int8_draws(gen, rows, cols, pad=0):
    return torch.randint(-127, 128, (rows, cols + pad), generator=gen, device="cuda", dtype=torch.int8)[:, :cols]


def generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


class Out:
    """rows x cols inside a buffer of 77s, `lead` elements before the first row and `pad` after each."""

    def __init__(self, rows, cols, dtype, pad, lead=0):
        self.buf = torch.full((rows * (cols + pad) + lead,), 77.0, dtype=TYPES[dtype], device="cuda")
        self.lead, self.pad, self.cols = lead, pad, cols
        self.view = self.buf[lead:].view(rows, cols + pad)[:, :cols]

    def beside_is_untouched(self):
        rows = self.buf[self.lead:].view(-1, self.cols + self.pad)
        return bool((self.buf[:self.lead] == 77).all() and (rows[:, self.cols:] == 77).all())


def off(got, want, bound, dtype):
    """How many elements are out of tolerance."""
    tol = bound + UNIT[dtype] * (want.abs() + bound) + TINY[dtype]
    return int((~((got.double() - want).abs() <= tol)).sum())


def act64(g, act):
    if act == lordba.ACT_SILU:
        return g * torch.sigmoid(g)
    return g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3))) / 2


# h and gate / up each with their own pad and lead; d_hidden mod 32 from 1 to 7, 0, and more.  14 x 17 tiles of 256 x 128: three
# or four a pair
@pytest.mark.parametrize("n,h_pad,h_lead,pre_pad,pre_lead", [
    (2052, 4, 0, 4, 0), (2049, 7, 0, 7, 0), (2055, 1, 0, 9, 0),      # all within the copy engine's reach
    (2052, 4, 0, 5, 0), (2112, 0, 0, 8, 1), (2052, 12, 0, 4, 3),     # h is, gate and up are not
    (2052, 5, 0, 4, 0), (2112, 8, 1, 0, 0),                          # gate and up are, h is not
    (2060, 4, 0, 4, 0), (2112, 0, 0, 0, 0), (2050, 1, 1, 1, 1)])
@pytest.mark.parametrize("dtype,act,adds", [("bf16", 0, False), ("f16", 1, True)])
def test_gated_forward_over_many_tiles(n, h_pad, h_lead, pre_pad, pre_lead, dtype, act, adds):
    T, K = 3500, 64
    gen = generator(n + h_pad)
    x, wg, wu = draws(gen, T, K, dtype), draws(gen, n, K, dtype, 0.2), draws(gen, n, K, dtype, 0.2)
    ga, ua = (draws(gen, T, n, dtype, 0.5, 3), draws(gen, T, n, dtype, 0.5, 3)) if adds else (None, None)
    g, u = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    eg, eu = (K * 2.0 ** -23 * (x.double().abs() @ w.double().abs().t()) for w in (wg, wu))
    if adds:
        g, u = g + ga.double(), u + ua.double()
        eg, eu = eg + 2.0 ** -23 * g.abs(), eu + 2.0 ** -23 * u.abs()
    a = act64(g, act)
    eh = 1.13 * eg * (u.abs() + eu) + a.abs() * eu + 2.0 ** -18 * (a * u).abs()
    first = None
    for save in (True, True, True, False):
        outs = [Out(T, n, dtype, h_pad, h_lead), Out(T, n, dtype, pre_pad, pre_lead), Out(T, n, dtype, pre_pad, pre_lead)]
        h, gate, up = (o.view for o in outs)
        lordba.gated_forward(x, wg, wu, h=h, act=act, gate_add=ga, up_add=ua, gate=gate if save else None, up=up if save else None)
        assert lordba.device_status() == 0
        assert all(o.beside_is_untouched() for o in outs)
        if first is None:
            assert off(gate, g, eg, dtype) == 0 and off(up, u, eu, dtype) == 0
            assert off(h, a * u, eh, dtype) == 0
            first = [t.clone() for t in (h, gate, up)]
        assert torch.equal(h, first[0])
        assert not save or (torch.equal(gate, first[1]) and torch.equal(up, first[2]))


# d_out mod 16 from 1 to 3 and mod 32 from 1 to 7; the pads make rows of whole 16 bytes, or not.  14 x 17 tiles of 256 x 256
@pytest.mark.parametrize("n,dtype,pad", [(4098, "f32", 2), (4097, "f32", 3), (4115, "f32", 1), (4099, "f32", 0), (4100, "f16", 4), (4097, "bf16", 7),
                                         (4103, "f16", 1), (4096, "bf16", 0), (4101, "f16", 0)])
def test_int8_linear_over_many_tiles(n, dtype, pad):
    T, K = 3500, 64
    gen = generator(n)
    x, w = int8_draws(gen, T, K), int8_draws(gen, n, K)
    s_x, s_w = (torch.randn(k, generator=gen, device="cuda").mul_(0.5).exp_().mul_(2.0 ** -8) for k in (T, n))
    want = (x.double() @ w.double().t()) * torch.outer(s_x.double(), s_w.double())
    first = None
    for _ in range(4):
        y = Out(T, n, dtype, pad)
        lordba.int8_linear(x, s_x, w, s_w, y.view)
        assert lordba.device_status() == 0 and y.beside_is_untouched()
        if first is None:
            assert off(y.view, want, 4 * 2.0 ** -24 * want.abs(), dtype) == 0
            first = y.view.clone()
        assert torch.equal(y.view, first)


@pytest.mark.parametrize("n,pad,save", [(2052, 4, True), (2049, 0, True), (2112, 0, False)])
def test_gated_forward_int8_over_many_tiles(n, pad, save):
    T, K = 3500, 128
    gen = generator(n)
    x, wg, wu = int8_draws(gen, T, K), int8_draws(gen, n, K), int8_draws(gen, n, K)
    s = [torch.randn(k, generator=gen, device="cuda").mul_(0.5).exp_().mul_(m) for k, m in ((T, 1.0), (n, 1.6e-5), (n, 1.6e-5))]
    g, u = ((x.double() @ w.double().t()) * torch.outer(s[0].double(), q.double()) for w, q in ((wg, s[1]), (wu, s[2])))
    a = act64(g, 0)
    eg, eu = 6 * 2.0 ** -24 * g.abs(), 6 * 2.0 ** -24 * u.abs()
    eh = 1.13 * eg * (u.abs() + eu) + a.abs() * eu + 2.0 ** -18 * (a * u).abs()
    first = None
    for _ in range(3):
        outs = [Out(T, n, "f16", pad) for _ in range(3)]
        h, gate, up = (o.view for o in outs)
        lordba.gated_forward(x, wg, wu, h=h, scales=tuple(s), gate=gate if save else None, up=up if save else None)
        assert lordba.device_status() == 0 and all(o.beside_is_untouched() for o in outs)
        if first is None:
            assert off(h, a * u, eh, "f16") == 0
            assert not save or (off(gate, g, eg, "f16") == 0 and off(up, u, eu, "f16") == 0)
            first = [o.view.clone() for o in outs]
        assert all(torch.equal(o.view, f) for o, f in zip(outs, first))


# dx of 16 x 17 tiles; both dW of 9 x 17 tiles each, one with its entries as two terms (up to 64 tokens)
@pytest.mark.parametrize("T,n,d_in,pad", [(4000, 64, 4100, 4), (4000, 72, 4097, 0), (96, 2052, 4100, 4), (40, 2052, 4100, 4), (130, 2056, 4103, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_gated_backward_over_many_tiles(T, n, d_in, pad, dtype):
    gen = generator(T + n)
    dh, gate, up = (draws(gen, T, n, dtype) for _ in range(3))
    x, wg, wu = draws(gen, T, d_in, dtype), draws(gen, n, d_in, dtype, 0.1), draws(gen, n, d_in, dtype, 0.1)
    first = None
    for _ in range(3):
        outs = [Out(T, d_in, dtype, pad), Out(n, d_in, dtype, pad), Out(n, d_in, dtype, pad)]
        dgate, dup, dx, dwg, dwu = lordba.gated_backward(dh, gate, up, x, wg, wu, dx=outs[0].view, dw_gate=outs[1].view, dw_up=outs[2].view)
        assert lordba.device_status() == 0 and all(o.beside_is_untouched() for o in outs)
        if first is None:
            dg, du, terms, eg, eu = dgate.double(), dup.double(), 1, 0.0, 0.0
            if T <= 64:            # the products' entries are the formula's, to the second term's rounding
                g, u, v = gate.double(), up.double(), dh.double()
                f = torch.sigmoid(g)
                dg, du, terms = v * u * f * (1 + g * (1 - f)), v * g * f, 2
                eg = 2.0 ** -18 * (v * u).abs() * 2.4 + UNIT[dtype] ** 2 * dg.abs() + TINY[dtype]
                eu = (2.0 ** -18 + UNIT[dtype] ** 2) * du.abs() + TINY[dtype]
            eg, eu = eg + 0 * dg, eu + 0 * du
            mg, mu = dg.abs() + eg, du.abs() + eu
            ag, au, ax = wg.double().abs(), wu.double().abs(), x.double().abs()
            err = terms * 2 * n * 2.0 ** -23 * (mg @ ag + mu @ au) + eg @ ag + eu @ au
            assert off(dx, dg @ wg.double() + du @ wu.double(), err, dtype) == 0
            assert off(dwg, dg.t() @ x.double(), terms * T * 2.0 ** -23 * (mg.t() @ ax) + eg.t() @ ax, dtype) == 0
            assert off(dwu, du.t() @ x.double(), terms * T * 2.0 ** -23 * (mu.t() @ ax) + eu.t() @ ax, dtype) == 0
            first = [o.view.clone() for o in outs]
        assert all(torch.equal(o.view, f) for o, f in zip(outs, first))
