"""Distillation where classes are masked by the lowest value of the logits' type, by another very low number, or by minus infinity:
a masked class has no chance and spoils nothing, wherever in the row it stands.

Bounds as in test_gpu_distill_offsets, of the classes that are not masked; a masked one's gradient is what the teacher leaves of it.
"""
import math

import numpy as np
import pytest
import torch

from paper_2605_24058_b200 import lordba
from test_gpu_block import TYPES
from test_gpu_distill_offsets import definition, within

pytestmark = pytest.mark.gpu

PLACES = {
    "first": lambda V: slice(0, V * 3 // 4),                     # whole threads' pieces, and the first rounds of a running maximum
    "last": lambda V: slice(V - 8, V),                           # a last piece
    "end": lambda V: slice(V // 3, V),
    "all but a few": lambda V: slice(5, V - 4),
}


def low(kind, dtype):
    return {"lowest": torch.finfo(TYPES[dtype]).min, "1e30": -1e30, "1e9": -1e9, "infinite": -math.inf}[kind]


def case(T, V, dtype, seed, spare):
    """Logits, the teacher's entries among the classes of `spare`, weights."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    z = (torch.randn(T, V, generator=gen, device="cuda") * 3).to(TYPES[dtype])
    ids = torch.stack([spare[torch.randperm(len(spare), generator=gen, device="cuda")[:5]] for _ in range(T)])
    return z, ids, torch.randn(T, 5, generator=gen, device="cuda") * 2, torch.rand(T, generator=gen, device="cuda") + 0.5


def everything(test):
    for mark in (pytest.mark.parametrize("place", sorted(PLACES)),
                 pytest.mark.parametrize("kind,dtype", [("lowest", "bf16"), ("lowest", "f16"), ("lowest", "f32"), ("1e30", "bf16"), ("1e30", "f32"), ("1e9", "bf16"), ("infinite", "bf16"),
                                                        ("infinite", "f32")]),
                 pytest.mark.parametrize("T,V", [(3, 512), (200, 512), (3, 4100), (3, 32000), (200, 32000), (700, 20000), (3, 140000), (200, 140000), (2, 600001)]),
                 pytest.mark.parametrize("tau", [1.0, 2.0, 0.5])):
        test = mark(test)
    return test


def masked_case(place, kind, dtype, T, V):
    """Logits, ids, teacher, weights, which classes are masked, and the ids among those that are not."""
    masked = torch.zeros(V, dtype=torch.bool, device="cuda")
    masked[PLACES[place](V)] = True
    z, ids, teacher, weight = case(T, V, dtype, V + T, (~masked).nonzero()[:, 0])
    z[:, masked] = low(kind, dtype)
    return z, ids, teacher, weight, masked, (torch.cumsum(~masked, 0) - 1)[ids]


@everything
def test_losses_beside_masked_classes(place, kind, dtype, T, V, tau):
    z, ids, teacher, weight, masked, left = masked_case(place, kind, dtype, T, V)
    loss, lse, _, tol_loss, tol_lse, _, _ = definition(z[:, ~masked], left, teacher, weight, tau)
    for got in (lordba.distill_loss(z, ids, teacher, tau, weight), lordba.distill_loss(z, ids, teacher, tau, weight, grad=True)):
        within(got[0], loss, tol_loss, "f32", "loss")
        within(got[1], lse, tol_lse, "f32", "lse")


throughout = lambda test: pytest.mark.parametrize("kind,dtype", [("lowest", "bf16"), ("lowest", "f16"), ("lowest", "f32"), ("1e30", "f32"), ("1e9", "bf16")])(
    pytest.mark.parametrize("T,V", [(3, 512), (200, 512), (200, 32000), (3, 140000), (200, 140000)])(test))


def even_case(kind, dtype, T, V):
    z, ids, teacher, weight = case(T, V, dtype, V + T, torch.arange(V, device="cuda"))
    z[:] = low(kind, dtype)
    return z, ids, teacher, weight


@throughout
def test_rows_masked_throughout_are_even(kind, dtype, T, V):
    """All classes at one very low number: each has the chance 1 / V."""
    z, ids, teacher, weight = even_case(kind, dtype, T, V)
    loss, lse, _, tol_loss, tol_lse, _, _ = definition(z, ids, teacher, weight, 1.0)
    for got in (lordba.distill_loss(z, ids, teacher, 1.0, weight), lordba.distill_loss(z, ids, teacher, 1.0, weight, grad=True)):
        within(got[0], loss, tol_loss, "f32", "loss")
        within(got[1], lse, tol_lse, "f32", "lse")


@everything
def test_gradients_beside_masked_classes(place, kind, dtype, T, V, tau):
    z, ids, teacher, weight, masked, left = masked_case(place, kind, dtype, T, V)
    _, _, dz, _, _, tol_dz, tol_back = definition(z[:, ~masked], left, teacher, weight, tau)
    step = lordba.distill_loss(z, ids, teacher, tau, weight, grad=True)
    back = lordba.distill_backward(weight, z, ids, teacher, step[1], tau)
    for g, tol in ((step[2], tol_dz), (back, tol_back)):
        within(g[:, ~masked], dz, tol, dtype, "dlogits")
        assert (g[:, masked] == 0).all()


@throughout
def test_gradients_of_rows_masked_throughout(kind, dtype, T, V):
    z, ids, teacher, weight = even_case(kind, dtype, T, V)
    _, _, dz, _, _, tol_dz, _ = definition(z, ids, teacher, weight, 1.0)
    _, lse, got = lordba.distill_loss(z, ids, teacher, 1.0, weight, grad=True)
    within(got, dz, tol_dz, dtype, "dlogits")
    # the way back knows lse in float32 alone, which has no room for log V beside such a number: the formula's value for the lse given
    back = lordba.distill_backward(weight, z, ids, teacher, lse)
    q = (z.double() - lse.double()[:, None]).exp()
    want = weight.double()[:, None] * q.scatter_add(1, ids, -teacher.double().softmax(1))
    # z - lse is rounded once (float16's is of some tens; the others' 0), the power's argument twice more
    within(back, want, weight.double()[:, None] * (q + 1) * 2.0 ** -18, dtype, "dlogits of distill_backward")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V", [(3, 512), (200, 32000), (200, 140000)])
def test_a_masked_class_of_the_teacher(dtype, T, V):
    """The teacher names a class that the student masks: a very large loss (float32 holds it), gradient -p there."""
    z, ids, teacher, weight = case(T, V, dtype, 7 * V + T, torch.arange(V // 2, V, device="cuda"))
    z[:, :V // 2] = -1e30
    ids[:, 2] = 7
    loss, lse, dz, tol_loss, tol_lse, tol_dz, _ = definition(z, ids, teacher, weight, 1.0)
    got = lordba.distill_loss(z, ids, teacher, 1.0, weight, grad=True)
    assert (loss > 1e20).all()
    within(got[0], loss, tol_loss, "f32", "loss")
    within(got[1], lse, tol_lse, "f32", "lse")
    within(got[2], dz, tol_dz, dtype, "dlogits")
