"""Distillation of long rows whose logits are equal, clipped or far from zero, against float64: what a running maximum over a
row's pieces could lose.

Tolerances, from the arithmetic.  A power of two has the argument (z - max) log2(e)/temperature, which is rounded three times
(the difference, the factor, the product), and an instruction good to 2^-22: a term is good to 2^-22 + |z - max|/temperature 2^-22 of
itself, a sum of them to that of the mean over its terms.  A thread adds at most V / 1024 terms one after the other (256 threads a row
or more, four sums each), then come trees of less than 32 additions, and a sum that meets a larger maximum is scaled once more, less than
32 times here.  E below is the sum of these; the logarithm adds 2^-23 of itself.  So log(sum) is good to E + log V 2^-23, however far
from zero the logits lie, and lse to that and three roundings of max / temperature and one of itself.  A probability that is not made from
lse: E + log V 2^-23 and the 2^-22 (1 + |z - max|/temperature) of its own power.  From lse: what lse is off, and three roundings of a number of its size.
"""
import math

import numpy as np
import pytest
import torch

from paper_2605_24058_b200 import lordba
from test_gpu_block import TINY, TYPES, UNIT

pytestmark = pytest.mark.gpu


def definition(z, ids, teacher, weight, tau):
    """(loss, lse, dz) and their bounds, and dz's from lse, in float64 on the device; ids all present and different."""
    z, teacher, weight = z.double(), teacher.double(), weight.double()
    top = z.max(1, keepdim=True).values
    s = (z - top) / tau
    e = s.exp()
    log_sum = e.sum(1).log()
    q = e / e.sum(1, keepdim=True)
    p = (teacher / tau).softmax(1)
    log_q, log_p = s.gather(1, ids) - log_sum[:, None], p.log()
    loss = weight * tau ** 2 * (p * (log_p - log_q)).sum(1)
    lse = top[:, 0] / tau + log_sum
    dz = (weight * tau)[:, None] * q.scatter_add(1, ids, -p)
    V = z.shape[1]
    E = 2.0 ** -22 * (1 + (q * s.abs()).sum(1)) + (V / 1024 + 64) * 2.0 ** -24 + 32 * 2.0 ** -21
    E_log = E + math.log(V) * 2.0 ** -23
    # the teacher's p: the exponential of a rounded quotient, over a sum
    off_p = p * (2.0 ** -20 + log_p.abs() * 2.0 ** -22)
    tol_loss = weight * tau ** 2 * ((p * (E_log[:, None] + (log_p.abs() + log_q.abs() + s.gather(1, ids).abs()) * 2.0 ** -22)).sum(1) + (off_p * (log_p - log_q).abs()).sum(1))
    tol_lse = E_log + 2.0 ** -22 * torch.maximum(top[:, 0].abs() / tau, lse.abs())
    around = torch.zeros_like(z).scatter_(1, ids, off_p)
    near = lambda by: (weight * tau)[:, None] * (q * (by[:, None] + 2.0 ** -22 * (1 + s.abs())) + around)
    return loss, lse, dz, tol_loss, tol_lse, near(E_log), near(tol_lse + 2.0 ** -22 * torch.maximum(top[:, 0].abs() / tau, lse.abs()))


def within(got, want, bound, dtype, what):
    off = (got.double() - want).abs()
    tol = bound + UNIT[dtype] * (want.abs() + bound) + TINY[dtype]
    bad = ~(off <= tol)
    assert not bad.any(), "%s: %d of %d off, worst %.3e times the bound" % (what, int(bad.sum()), bad.numel(), float((off / tol).max()))


def logits(kind, T, V, offset, dtype, gen):
    z = torch.randn(T, V, generator=gen, device="cuda") * 3
    if kind == "equal":
        z.zero_()
    elif kind == "clipped":
        z.clamp_(max=0.0)                 # half of the row at its maximum
    elif kind == "rising":
        z = torch.linspace(-3, 3, V, device="cuda").expand(T, V) + 0.01 * z
    return (z + offset).to(TYPES[dtype])


def everything(test):
    for mark in (pytest.mark.parametrize("kind", ["equal", "clipped", "spread", "rising"]), pytest.mark.parametrize("dtype", ["f32", "bf16"]),
                 pytest.mark.parametrize("T,V,tau", [(3, 131072, 1.0), (3, 300001, 1.0), (2, 1000003, 0.7), (160, 131072, 1.0), (160, 160000, 2.0), (150, 262144, 0.7)]),
                 pytest.mark.parametrize("offset", [0.0, 100.0, -1000.0, 1000.0])):
        test = mark(test)
    return test


def case(kind, dtype, T, V, tau, offset):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(V + T)
    z = logits(kind, T, V, offset, dtype, gen)
    ids = torch.stack([torch.randperm(V, generator=gen, device="cuda")[:9] for _ in range(T)])
    teacher = torch.randn(T, 9, generator=gen, device="cuda") * 2
    weight = torch.rand(T, generator=gen, device="cuda") + 0.5
    return z, ids, teacher, float(np.float32(tau)), weight


@everything
def test_losses_of_offset_rows(kind, dtype, T, V, tau, offset):
    z, ids, teacher, tau, weight = case(kind, dtype, T, V, tau, offset)
    loss, lse, _, tol_loss, tol_lse, _, _ = definition(z, ids, teacher, weight, tau)
    for got in (lordba.distill_loss(z, ids, teacher, tau, weight), lordba.distill_loss(z, ids, teacher, tau, weight, grad=True)):
        within(got[0], loss, tol_loss, "f32", "loss")
        within(got[1], lse, tol_lse, "f32", "lse")


@everything
def test_gradients_of_offset_rows(kind, dtype, T, V, tau, offset):
    z, ids, teacher, tau, weight = case(kind, dtype, T, V, tau, offset)
    _, lse, dz, _, _, tol_dz, tol_back = definition(z, ids, teacher, weight, tau)
    within(lordba.distill_loss(z, ids, teacher, tau, weight, grad=True)[2], dz, tol_dz, dtype, "dlogits")
    lse = lordba.distill_loss(z, ids, teacher, tau, weight)[1]
    within(lordba.distill_backward(weight, z, ids, teacher, lse, tau), dz, tol_back, dtype, "dlogits of distill_backward")
