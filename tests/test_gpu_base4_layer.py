"""The operators around a 4-bit base, run together as the example runs them: a training step of an adapted attention layer
that learns from a teacher, against the same layer in float32."""
import importlib.util
import os

import pytest
import torch

from paper_2605_24058_b200 import lordba
from test_gpu_block import clean

pytestmark = pytest.mark.gpu


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "distilled_attention.py")
    spec = importlib.util.spec_from_file_location("distilled_attention", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


# Of few tokens, of some tens, and of many: every way that the products go.
@pytest.mark.parametrize("tokens,d_model,heads,key_heads,d,vocab,top", [(3, 256, 4, 2, 64, 1000, 5), (24, 320, 4, 1, 80, 777, 16), (90, 512, 4, 4, 128, 2048, 64),
                                                                         (300, 384, 6, 2, 64, 1501, 32)])
def test_the_distilled_layer_of_the_example(tokens, d_model, heads, key_heads, d, vocab, top):
    """24 bfloat16 roundings (2^-9 each in the mean, of independent signs, so that their sum leaves room for what the softmaxes
    make of them) lie between the two: eight results on the way to the logits, nine gradients on the way back, and the
    weights of three products in either direction; dw_q and dw_k are measured by their terms."""
    errors = example().run(tokens, d_model, heads, key_heads, d, vocab, top, 8)
    assert set(errors) == {"loss", "dx", "dw_q", "dw_k"}
    assert all(e < 24 * 2.0 ** -9 for e in errors.values()), errors
    clean()


@pytest.mark.parametrize("tokens", [1, 24, 90])
def test_a_captured_step_repeats(tokens):
    """The layer's own calls in a CUDA graph: replayed on new inputs, twice, with the bits of the calls one by one."""
    module = example()
    layer = module.Layer(256, 4, 2, 64, 500, 8)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    draw = lambda: torch.randn(tokens, 256, generator=gen, device="cuda").to(torch.bfloat16)
    positions = torch.arange(tokens, device="cuda")
    ids = torch.randint(0, 500, (tokens, 9), generator=gen, device="cuda")
    teacher = torch.randn(tokens, 9, generator=gen, device="cuda")
    x = draw()

    def step():
        qkv = layer.product(x, layer.qkv)
        q, k, _ = layer.parts(qkv)
        q_out, k_out = lordba.norm_rope(q, k, positions, layer.inv_freq, layer.w_q, layer.w_k)
        logits = layer.product(q_out.flatten(1), layer.head)
        loss, lse, dlogits = lordba.distill_loss(logits, ids, teacher, 1.5, dlogits=logits)
        dq_out = layer.turn_back(dlogits, layer.head, 256).unflatten(1, (-1, 64))
        dqkv = torch.zeros_like(qkv)
        dq, dk, _ = layer.parts(dqkv)
        _, _, dw_q, dw_k = lordba.norm_rope_backward(dq_out, k_out, q, k, positions, layer.inv_freq, layer.w_q, layer.w_k, dq=dq, dk=dk)
        return loss, lse, dlogits, dw_q, dw_k, layer.turn_back(dqkv, layer.qkv, 256)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(2):
        x.copy_(draw())
        want = [t.clone() for t in step()]
        for _ in range(2):
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(held, want))
    clean()
