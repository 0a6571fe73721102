"""GPU parity of the distillation loss and its gradient against a float64 implementation written here.

Tolerances, from the arithmetic (u as in test_gpu_block).  An exponential is a power of two of an argument that is good to
2^-24 of the numbers it is the difference of, times an instruction good to 2^-22; a row's sum adds at most V / 128 of them one
after the other, then trees.  With S the largest |logit| / temperature (and lse) of a row, a probability is good to
E = 2^-20 + 4 S 2^-23 + V 2^-31 of itself and lse to E.  A p of the teacher's is the exponential of a quotient that is rounded
once, 2^-24 of |log p + log total| <= |log p| + log 256, over a sum: good to 2^-20 + |log p| 2^-23 of itself.  The loss: each
of its terms p (log p - log q) is good to p (|log p| + |log q| + 1) (2^-20 + E).
"""
import math

import numpy as np
import pytest
import torch

from paper_2605_24058_b200 import lordba
from test_gpu_block import TINY, TYPES, UNIT, f64, target, untouched

pytestmark = pytest.mark.gpu


def definition(z, ids, teacher, weight, tau):
    """(loss, lse, dz, bounds of the three) in float64."""
    T, V = z.shape
    z = z / tau
    lse = np.log(np.exp(z - z.max(1, keepdims=True)).sum(1)) + z.max(1)
    here = (ids >= 0) & (ids < V)
    v = np.where(here, teacher / tau, -np.inf)
    most = v.max(1, keepdims=True)
    e = np.where(v > -np.inf, np.exp(v - np.where(np.isfinite(most), most, 0.0)), 0.0)
    total = e.sum(1, keepdims=True)
    p = e / np.where(total > 0, total, 1.0)
    log_p = np.where(p > 0, np.log(np.where(p > 0, p, 1.0)), 0.0)
    log_q = np.where(p > 0, np.take_along_axis(z, np.where(here, ids, 0), 1) - lse[:, None], 0.0)
    alive = (weight != 0) & (total[:, 0] > 0)
    loss = np.where(alive, weight * tau ** 2 * (p * (log_p - log_q)).sum(1), 0.0)
    q = np.exp(z - lse[:, None])
    dense, off = np.zeros_like(z), np.zeros_like(z)
    for t in range(T):
        np.add.at(dense[t], ids[t][here[t]], p[t][here[t]])
        np.add.at(off[t], ids[t][here[t]], (p * (2.0 ** -20 + np.abs(log_p) * 2.0 ** -23))[t][here[t]])
    dz = np.where(alive[:, None], (q - dense) * (weight * tau)[:, None], 0.0)
    finite = np.where(np.isfinite(z), np.abs(z), 0.0)
    E = 2.0 ** -20 + 4 * np.maximum(finite.max(1), np.abs(lse)) * 2.0 ** -23 + V * 2.0 ** -31
    size = np.where(np.isfinite(log_q), np.abs(log_q), 0.0) + np.abs(log_p) + 1
    tol_loss = np.abs(weight) * tau ** 2 * (p * size).sum(1) * (2.0 ** -20 + E)
    return loss, lse, dz, tol_loss, E, (np.abs(weight) * tau)[:, None] * (E[:, None] * q + off)


def within(got, want, bound, dtype, what):
    got = f64(got)
    tol = bound + UNIT[dtype] * (np.abs(want) + bound) + TINY[dtype]
    bad = ~((np.abs(got - want) <= tol) | (got == want))
    assert got.shape == want.shape and not bad.any(), "%s: %d of %d off, first at %s: got %r want %r tol %r" % (
        what, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0], np.broadcast_to(tol, bad.shape)[bad][0])


class Case:
    def __init__(self, rng, T, V, top, dtype, pad=0, lead=0, wide=False, teacher="f32", weights=True):
        z = torch.from_numpy((rng.standard_normal(T * (V + pad) + lead) * 3).astype(np.float32)).to(TYPES[dtype]).cuda()
        self.logits = z[lead:].view(T, V + pad)[:, :V]
        self.ids_np = np.stack([rng.choice(V, top, replace=top > V) for _ in range(T)])
        if top > 3:
            self.ids_np[::3, top // 2] = -1                        # absent ones, and one that stands there twice
            self.ids_np[1::3, 1] = self.ids_np[1::3, 0]
            self.ids_np[::4, 2] = V
        self.ids = torch.from_numpy(self.ids_np.astype(np.int64 if wide else np.int32)).cuda()
        self.teacher = torch.from_numpy((rng.standard_normal((T, top)) * 2 + 4).astype(np.float32)).to(TYPES[teacher]).cuda()
        w = rng.uniform(0.5, 2.0, T).astype(np.float32)
        w[3::5] = 0
        self.weight = torch.from_numpy(w).cuda() if weights else None
        self.weight_np = w.astype(np.float64) if weights else np.ones(T)

    def definition(self, tau):
        return definition(f64(self.logits), self.ids_np, f64(self.teacher), self.weight_np, float(np.float32(tau)))


SIZES = [  # T, V, top, pad, lead
    (1, 1, 1, 0, 0), (1, 8, 3, 0, 0), (3, 33, 5, 0, 0), (2, 1000, 20, 5, 1), (1, 32000, 64, 0, 0), (7, 32003, 20, 1, 0), (40, 1023, 256, 1, 0), (5, 4096, 100, 8, 0),
    (64, 2050, 33, 0, 3), (150, 5000, 8, 0, 0), (9, 50257, 50, 0, 0), (3, 131072, 32, 0, 0), (160, 33000, 16, 0, 0), (2, 300001, 7, 0, 0), (1, 700000, 10, 0, 0), (300, 128, 4, 0, 0),
    (150, 120000, 16, 5, 1), (600, 9001, 8, 0, 0)]


@pytest.mark.parametrize("T,V,top,pad,lead", SIZES)
@pytest.mark.parametrize("dtype,wide,teacher,tau,weights", [("bf16", True, "bf16", 1.0, True), ("f16", False, "f32", 2.0, False), ("f32", True, "f16", 0.7, True)])
def test_distill(T, V, top, pad, lead, dtype, wide, teacher, tau, weights):
    c = Case(np.random.default_rng(V + T), T, V, top, dtype, pad, lead, wide, teacher, weights)
    loss, lse, dz, tol_loss, tol_lse, tol_dz = c.definition(tau)
    args = (c.ids, c.teacher, tau)
    got = lordba.distill_loss(c.logits, *args, weight=c.weight)
    assert got[2] is None
    within(got[0], loss, tol_loss, "f32", "loss")
    within(got[1], lse, tol_lse, "f32", "lse")
    buf, out = target(T, V, dtype, pad, lead)
    step = lordba.distill_loss(c.logits, *args, weight=c.weight, dlogits=out)
    # the loss alone adds a row's exponentials in another order: either is within the bound of any order
    within(step[0], loss, tol_loss, "f32", "loss with the gradient")
    within(step[1], lse, tol_lse, "f32", "lse with the gradient")
    assert step[2] is out
    within(out, dz, tol_dz, dtype, "dlogits")
    untouched(buf, T, V, pad, lead)
    made = lordba.distill_loss(c.logits, *args, weight=c.weight, grad=True)[2]
    assert torch.equal(made, out)
    # the way back in a call of its own: lse is rounded once more on its way
    up = c.weight if weights else torch.ones(T, device="cuda")
    buf, out = target(T, V, dtype, pad, lead)
    lordba.distill_backward(up, c.logits, c.ids, c.teacher, got[1], tau, dlogits=out)
    within(out, dz, tol_dz, dtype, "dlogits of distill_backward")
    untouched(buf, T, V, pad, lead)
    # over the logits
    for call in (lambda z: lordba.distill_loss(z, *args, weight=c.weight, dlogits=z), lambda z: lordba.distill_backward(up, z, c.ids, c.teacher, got[1], tau, dlogits=z)):
        buf = torch.full((T * (V + pad) + lead,), 77.0, dtype=TYPES[dtype], device="cuda")
        z = buf[lead:].view(T, V + pad)[:, :V]
        z.copy_(c.logits)
        call(z)
        within(z, dz, tol_dz, dtype, "dlogits over the logits")
        untouched(buf, T, V, pad, lead)


@pytest.mark.parametrize("V", [50, 33000, 140000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_anything_to_learn(V, dtype):
    """Weight 0, no entry, entries of minus infinity alone: loss and gradient 0 whatever the logits hold."""
    T, top = 6, 4
    z = torch.randn(T, V, device="cuda").to(TYPES[dtype])
    z[1, 3], z[2, 7], z[4] = math.nan, math.inf, -math.inf
    ids = torch.arange(top, device="cuda").repeat(T, 1)
    teacher = torch.randn(T, top, device="cuda")
    weight = torch.ones(T, device="cuda")
    weight[1] = weight[4] = 0
    ids[2], teacher[3] = -1, -math.inf
    loss, lse, dz = lordba.distill_loss(z, ids, teacher, weight=weight, grad=True)
    assert (loss[1:5] == 0).all() and (dz[1:5] == 0).all() and torch.isfinite(loss).all() and torch.isfinite(dz).all()
    assert loss[0] != 0 and (dz[0] != 0).any() and torch.isfinite(lse[[0, 3, 5]]).all() and lse[4] == -math.inf
    again = lordba.distill_backward(weight, z, ids, teacher, lse)
    assert (again[1:5] == 0).all() and torch.isfinite(again).all()


@pytest.mark.parametrize("V", [64, 40000])
def test_infinite_logits(V):
    T, top = 5, 3
    rng = np.random.default_rng(V)
    z = torch.from_numpy(rng.standard_normal((T, V)).astype(np.float32)).cuda()
    ids = torch.tensor([[1, 5, 9]] * T).cuda()
    teacher = torch.tensor([[1.0, 0.5, -math.inf]] * T).cuda()
    z[0, 20:40] = -math.inf               # masked classes, not among the teacher's
    z[1, 9] = -math.inf                   # one of the teacher's, with no chance there
    z[2, 5] = -math.inf                   # one of the teacher's that the student rules out
    z[3, 30] = math.inf
    z[4, 30] = math.nan
    loss, lse, dz = lordba.distill_loss(z, ids, teacher, grad=True)
    want = definition(f64(z)[:2], ids.cpu().numpy()[:2], f64(teacher)[:2], np.ones(2), 1.0)
    within(loss[:2], want[0], want[3], "f32", "loss")
    within(lse[:2], want[1], want[4], "f32", "lse")
    within(dz[:2], want[2], want[5], "f32", "dlogits")
    assert (dz[0, 20:40] == 0).all() and loss[2] == math.inf and torch.isfinite(dz[2]).all()
    assert torch.isnan(loss[3:]).all() and torch.isnan(dz[4]).all() and torch.isnan(dz[3, 30])
    teacher[0, 0] = math.nan
    loss, _, dz = lordba.distill_loss(z, ids, teacher, grad=True)
    assert torch.isnan(loss[0]) and torch.isnan(dz[0, 1]) and torch.isfinite(loss[1])


def test_gradient_is_a_difference():
    """Along a direction, central differences in float32: the third derivative of a log-sum along v is below 6 max|v|^3, and two
    losses are good to the tolerance of the loss."""
    rng = np.random.default_rng(8)
    c = Case(rng, 6, 700, 9, "f32")
    v = torch.from_numpy(rng.standard_normal((6, 700)).astype(np.float32)).cuda()
    tau, h = 2.0, 2.0 ** -5
    f = lambda z: lordba.distill_loss(z, c.ids, c.teacher, tau, weight=c.weight)[0].double()
    dz = lordba.distill_loss(c.logits, c.ids, c.teacher, tau, weight=c.weight, grad=True)[2]
    along = (f(c.logits + h * v) - f(c.logits - h * v)) / (2 * h)
    tol = h * h / 6 * 6 * float(v.abs().max()) ** 3 * f64(c.weight) + c.definition(tau)[3] / h + 1e-6
    assert (np.abs(f64(along) - f64((dz.double() * v.double()).sum(1))) <= tol).all()


def test_rows_far_apart():
    """Offsets that pass 32 bits."""
    far, V = (1 << 30) + 8, 1000
    big = torch.zeros(2 * far + V, dtype=torch.bfloat16, device="cuda")
    z = big.as_strided((3, V), (far, 1))
    z.copy_(torch.randn(3, V, device="cuda"))
    ids, teacher = torch.arange(5, device="cuda").repeat(3, 1), torch.randn(3, 5, device="cuda")
    want = lordba.distill_loss(z.contiguous(), ids, teacher, grad=True)
    got = lordba.distill_loss(z, ids, teacher, dlogits=z)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("V", [3000, 80000])
def test_streams_graphs_and_repeats(V):
    c = Case(np.random.default_rng(V), 50, V, 16, "bf16", wide=True)
    call = lambda **kw: lordba.distill_loss(c.logits, c.ids, c.teacher, 2.0, weight=c.weight, **kw)
    want = call(grad=True)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(call(grad=True), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(grad=True, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    outs = [torch.zeros_like(t) for t in want]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(loss=outs[0], lse=outs[1], dlogits=outs[2])
    for _ in range(2):
        for t in outs:
            t.zero_()
        g.replay()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_refusals():
    z = torch.randn(4, 100, device="cuda")
    ids, teacher = torch.arange(8, device="cuda").repeat(4, 1), torch.randn(4, 8, device="cuda")
    call = lambda z=z, ids=ids, teacher=teacher, tau=1.0, **kw: lordba.distill_loss(z, ids, teacher, tau, **kw)
    assert call()[0].shape == (4,)
    for wrong, error in [(dict(z=z[0]), ValueError), (dict(z=z.t()), ValueError), (dict(z=z.int()), TypeError), (dict(ids=ids.float()), TypeError), (dict(ids=ids[:3]), ValueError),
                         (dict(teacher=teacher[:, :7]), ValueError), (dict(teacher=teacher.double()), TypeError), (dict(z=z.cpu()), ValueError),
                         (dict(weight=torch.ones(3, device="cuda")), TypeError), (dict(weight=torch.ones(4, device="cuda").double()), TypeError),
                         (dict(dlogits=z.half()), TypeError), (dict(lse=torch.empty(5, device="cuda")), TypeError), (dict(tau="1"), TypeError)]:
        with pytest.raises(error):
            call(**wrong)
    loss = torch.empty(4, device="cuda")
    for wrong in (dict(tau=0.0), dict(tau=-1.0), dict(tau=math.nan), dict(loss=loss, lse=loss), dict(ids=ids[:, :0], teacher=teacher[:, :0]),
                  dict(ids=torch.zeros(4, 257, dtype=torch.int32, device="cuda"), teacher=torch.zeros(4, 257, device="cuda"))):
        with pytest.raises(lordba.LordbaError):
            call(**wrong)
    with pytest.raises(RuntimeError, match="gradient"):
        call(z=z.clone().requires_grad_(True))
    with pytest.raises(TypeError):
        lordba.distill_backward(torch.ones(3, device="cuda"), z, ids, teacher, loss)
    assert call(z=z[:0], ids=ids[:0], teacher=teacher[:0], grad=True)[2].shape == (0, 100)
