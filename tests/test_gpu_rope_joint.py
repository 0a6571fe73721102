"""Norm and rotation where a joint buffer holds each head's query, key and value side by side: results in place of the inputs, and
gradients in a joint buffer, with the values left as they are.  Same bits as from and into tensors of their own that are aligned alike."""
import numpy as np
import pytest
import torch

from paper_2605_24058_b200 import lordba
from test_gpu_block import TYPES
from test_gpu_rope import frequencies

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,heads,d,R,dtype", [(1, 1, 64, 64, "bf16"), (1, 5, 128, 128, "bf16"), (33, 6, 128, 128, "bf16"), (70, 3, 80, 40, "f32"), (200, 12, 64, 32, "f16"), (9, 2, 256, 256, "f32")])
def test_in_turns(T, heads, d, R, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    joint = torch.randn(T, heads, 3, d, generator=gen, device="cuda").to(TYPES[dtype])
    grads = torch.randn(T, heads, 2, d, generator=gen, device="cuda").to(TYPES[dtype])
    pos, inv = torch.arange(T, device="cuda") + 7, torch.from_numpy(frequencies(R)).cuda()
    w = [torch.rand(d, generator=gen, device="cuda") + 0.5 for _ in range(2)]
    q, k, v = (joint[:, :, i] for i in range(3))
    want = lordba.norm_rope(q, k, pos, inv, *w)
    back = lordba.norm_rope_backward(grads[:, :, 0], grads[:, :, 1], q, k, pos, inv, *w)
    dj = torch.full_like(joint, 77.0)
    got = lordba.norm_rope_backward(grads[:, :, 0], grads[:, :, 1], q, k, pos, inv, *w, dq=dj[:, :, 0], dk=dj[:, :, 1])
    assert torch.equal(dj[:, :, 0], back[0]) and torch.equal(dj[:, :, 1], back[1]) and (dj[:, :, 2] == 77).all()
    assert torch.equal(got[2], back[2]) and torch.equal(got[3], back[3])
    kept = v.clone()
    lordba.norm_rope(q, k, pos, inv, *w, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v, kept)
    with pytest.raises(lordba.LordbaError):
        lordba.norm_rope(q, k, pos, inv, *w, q_out=k, k_out=q)
