"""Distillation right behind the kernel that makes its logits, and right before one that reads its gradient: the same bits as with a
wait for the device in between, for rows that do their teacher's part themselves and for many, called and replayed."""
import numpy as np
import pytest
import torch

from paper_2605_24058_b200 import lordba
from test_gpu_block import clean, matrix
from test_gpu_int4 import Weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,d,V,grad", [(100, 256, 5000, True), (300, 256, 5000, True), (300, 256, 5000, False), (300, 128, 70001, True), (300, 128, 70000, False), (2000, 512, 1003, True)])
@pytest.mark.parametrize("in_place", [False, True])
def test_between_a_product_and_its_gradient(T, d, V, grad, in_place):
    rng = np.random.default_rng(T + V)
    xs = [matrix(rng, T, d, "bf16")[0] for _ in range(3)]
    w = Weights(rng, V, d, 64, True, "bf16", gain=8.0)
    ids = torch.from_numpy(rng.integers(0, V, (T, 16))).cuda()
    teacher = torch.from_numpy(rng.standard_normal((T, 16)).astype(np.float32)).cuda()
    logits, dz = torch.empty(T, (V + 7) // 8 * 8, dtype=torch.bfloat16, device="cuda")[:, :V], None
    if grad:
        dz = logits if in_place else torch.empty_like(logits)
    loss, lse, dx = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty(T, d, dtype=torch.bfloat16, device="cuda")

    def run(x, between):
        lordba.int4_linear(x, w.q, w.scale, w.zero, 64, y=logits)
        between()
        lordba.distill_loss(logits, ids, teacher, 2.0, loss=loss, lse=lse, dlogits=dz)
        between()
        if not grad:
            return [loss, lse]
        lordba.int4_linear_backward(dz, w.q, w.scale, d, w.zero, 64, dx=dx)
        return [loss, lse, dz, dx]

    wants = []
    for x in xs:
        wants.append([t.clone() for t in run(x, torch.cuda.synchronize)])
    for _ in range(3):
        for x, want in zip(xs, wants):
            assert all(torch.equal(a, b) for a, b in zip(run(x, lambda: None), want))
    taken = xs[0].clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = run(taken, lambda: None)
    for _ in range(3):
        for x, want in zip(xs, wants):
            taken.copy_(x)
            g.replay()
            assert all(torch.equal(a, b) for a, b in zip(outs, want))
    clean()
