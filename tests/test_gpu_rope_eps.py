"""Gradients of norm and rotation without an epsilon, where a step of a warp has room for more heads than there are: what no head
fills adds nothing to the sums of dw.  Tolerances as in test_gpu_rope."""
import numpy as np
import pytest
import torch

from paper_2605_24058_b200 import lordba
from test_gpu_block import TYPES, f64
from test_gpu_rope import backward, check, forward, frequencies, heads

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hk", [(1, 0), (2, 1), (3, 1), (5, 2), (6, 3), (4, 4), (33, 5)])
@pytest.mark.parametrize("d,R,interleaved", [(64, 64, False), (128, 128, False), (256, 256, True), (128, 64, False), (80, 80, True), (24, 16, False), (33, 20, False), (16, 0, False)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 37])
def test_no_epsilon(hq, hk, d, R, interleaved, dtype, T):
    rng = np.random.default_rng(hq * 100 + d)
    inv, pos = frequencies(R), rng.integers(0, 5000, T)
    n = max(hk, 1)
    (q, vq), (k, vk), (gq, vgq), (gk, vgk) = (heads(rng, T, h, d, dtype) for h in (hq, n, hq, n))
    w, v = [], []
    for _ in range(2):
        w.append(torch.from_numpy((1 + 0.3 * rng.standard_normal(d)).astype(np.float32)).to(TYPES[dtype]).cuda())
        v.append(f64(w[-1]))
    keys, dkeys = (k, gk) if hk else (None, None)
    args = (torch.from_numpy(pos).cuda(), torch.from_numpy(inv).cuda(), w[0], w[1] if hk else None)
    E = (d + 64) * 2.0 ** -22
    out = lordba.norm_rope(q, keys, *args, eps=0.0, interleaved=interleaved)
    got = lordba.norm_rope_backward(gq, dkeys, q, keys, *args, eps=0.0, interleaved=interleaved)
    for i, (g, x, h) in enumerate([(vgq, vq, hq), (vgk, vk, hk)][:2 if hk else 1]):
        want, size = forward(x, v[i], pos, inv, 0.0, True, interleaved)
        check(out[i], want, E * size, dtype, "qk"[i])
        dx, big, dw, dbig = backward(g, x, v[i], pos, inv, 0.0, True, interleaved)
        check(got[i], dx, E * big, dtype, "d" + "qk"[i])
        check(got[2 + i], dw, (E + T * h * 2.0 ** -24) * dbig, "f32", "dw")
