"""An attention layer whose projections are 4-bit and whose adapters learn from a teacher's top logits.

    qkv = W_qkv x  (+ adapters on the query and the key part)      4-bit weights, one joint product
    q, k = rotate(norm(q)), rotate(norm(k))                         slices of qkv, read in place
    y = x + W_o attention(q, k, v)  (+ adapter)
    loss = sum over tokens of weight * divergence of softmax(W_head y) from the teacher's

The forward pass of a few tokens is what serving runs.  A training step gets the gradient of the logits with the loss, and
brings it back through the frozen 4-bit projections, the adapters' adjoints, the rotation and the norms, whose
weights learn.  Attention itself is plain torch here.

    python examples/distilled_attention.py [--tokens T] [--d-model D] [--vocab V] [--top N] [--rank R]

prints how far the loss and the gradients are from the same layer in plain float32 torch.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from examples.adapted_feed_forward import Adapter  # noqa: E402
from paper_2605_24058_b200 import lordba  # noqa: E402


def attention(q, k, v):
    """Causal attention of (T, heads, d) queries and (T, key heads, d) keys and values, in float32."""
    share = q.shape[1] // k.shape[1]
    k, v = (t.float().repeat_interleave(share, 1) for t in (k, v))
    s = torch.einsum("thd,shd->hts", q.float(), k) / q.shape[2] ** 0.5
    later = torch.ones(s.shape[1:], dtype=torch.bool, device=s.device).triu(1)
    return torch.einsum("hts,shd->thd", s.masked_fill(later, float("-inf")).softmax(-1), v).flatten(1)


class Layer:
    def __init__(self, d_model, heads, key_heads, d, vocab, rank, group=64, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.heads, self.key_heads, self.d, self.d_model, self.group = heads, key_heads, d, d_model, group
        rows = (heads + 2 * key_heads) * d
        weight = lambda a, b: torch.randn(a, b, generator=gen, device="cuda") / b ** 0.5
        # once: the base in 4 bits, a scale and a zero point for every `group` columns of a row
        self.qkv, self.out, self.head = (lordba.int4_quantize(weight(a, b), group, zeros=True, dtype=torch.bfloat16)
                                         for a, b in ((rows, d_model), (d_model, heads * d), (vocab, d_model)))
        adapter = lambda a, b: Adapter(a, b, rank, gen, 0.5)
        self.on_q, self.on_k, self.on_out = adapter(d_model, heads * d), adapter(d_model, key_heads * d), adapter(heads * d, d_model)
        self.w_q, self.w_k = (1 + 0.2 * torch.randn(d, generator=gen, device="cuda") for _ in range(2))
        self.inv_freq = 10000.0 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float32) / d)

    def product(self, x, w):
        return lordba.int4_linear(x, w[0], w[1], w[2], self.group)

    def turn_back(self, dy, w, d_in):
        return lordba.int4_linear_backward(dy, w[0], w[1], d_in, w[2], self.group)

    def parts(self, qkv):
        """Queries, keys and values as views (T, heads, d) of the joint projection's output or of its gradient."""
        h, k, d = self.heads, self.key_heads, self.d
        return [t.unflatten(1, (-1, d)) for t in qkv.split((h * d, k * d, k * d), 1)]

    def forward(self, x, positions):
        """logits, and what the backward pass needs."""
        qkv = self.product(x, self.qkv)
        q, k, v = self.parts(qkv)
        self.on_q.add_to(x, q.flatten(1))
        self.on_k.add_to(x, k.flatten(1))
        q_out, k_out = lordba.norm_rope(q, k, positions, self.inv_freq, self.w_q, self.w_k)
        a = attention(q_out, k_out, v).to(x.dtype)
        o = self.product(a, self.out)
        self.on_out.add_to(a, o)
        return self.product(x + o, self.head), (qkv, q_out, k_out)

    def backward(self, dlogits, saved, positions):
        """Gradients of x, w_q and w_k.  dlogits is what distill_loss left."""
        qkv, q_out, k_out = saved
        q, k, v = self.parts(qkv)
        dy = self.turn_back(dlogits, self.head, self.d_model)
        da = self.turn_back(dy, self.out, self.heads * self.d)
        self.on_out.add_adjoint_to(dy, da)
        with torch.enable_grad():
            leaves = [t.detach().requires_grad_(True) for t in (q_out, k_out, v)]
            dq_out, dk_out, dv = torch.autograd.grad(attention(*leaves), leaves, da.float())
        dqkv = torch.empty_like(qkv)
        dq, dk, dv_part = self.parts(dqkv)
        dv_part.copy_(dv)
        _, _, dw_q, dw_k = lordba.norm_rope_backward(dq_out.contiguous(), dk_out.contiguous(), q, k, positions, self.inv_freq, self.w_q,
                                                     self.w_k, dq=dq, dk=dk)
        dx = self.turn_back(dqkv, self.qkv, self.d_model)
        self.on_q.add_adjoint_to(dq.flatten(1), dx)
        self.on_k.add_adjoint_to(dk.flatten(1), dx)
        return dx + dy, dw_q, dw_k

    def step(self, x, positions, ids, teacher, weight, temperature):
        """(the tokens' losses, gradients of their sum to x, w_q and w_k)"""
        logits, saved = self.forward(x, positions)
        loss, _, dlogits = lordba.distill_loss(logits, ids, teacher, temperature, weight, dlogits=logits)
        return (loss,) + self.backward(dlogits, saved, positions)

    # ---- the same in plain float32 torch ----------------------------------------------------------------------
    def plain_step(self, x, positions, ids, teacher, weight, temperature):
        """As step, with the gradients of w_q and w_k for every token and head (their sums are the gradients)."""
        qkv, out, head = (lordba.int4_dequantize(w[0], w[1], d, w[2], self.group).float()
                          for w, d in ((self.qkv, self.d_model), (self.out, self.heads * self.d), (self.head, self.d_model)))
        x = x.float().requires_grad_(True)
        q, k, v = self.parts(x @ qkv.t())
        q = q + (x @ self.on_q.dense().t()).unflatten(1, (-1, self.d))
        k = k + (x @ self.on_k.dense().t()).unflatten(1, (-1, self.d))
        w_q, w_k = (w.expand(t.shape).clone().requires_grad_(True) for w, t in ((self.w_q, q), (self.w_k, k)))
        angle = positions.double()[:, None, None] * self.inv_freq.double()
        cos, sin = angle.cos().float(), angle.sin().float()

        def turned(t, w):
            n = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6) * w
            a, b = n.chunk(2, -1)
            return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)

        a = attention(turned(q, w_q), turned(k, w_k), v)
        logits = (x + a @ out.t() + a @ self.on_out.dense().t()) @ head.t()
        p = (teacher / temperature).softmax(-1)
        picked = (logits / temperature).log_softmax(-1).gather(1, ids)
        loss = weight * temperature ** 2 * (p * (p.log() - picked)).sum(-1)
        loss.sum().backward()
        return loss.detach(), x.grad, w_q.grad, w_k.grad


def run(tokens, d_model, heads, key_heads, d, vocab, top, rank, temperature=2.0, seed=1):
    """Relative errors (2-norm) of a step's losses and gradients; those of w_q and w_k, which are sums of terms of either
    sign, relative to the root of the sum of the terms' squares."""
    layer = Layer(d_model, heads, key_heads, d, vocab, rank, seed=seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 1)
    x = torch.randn(tokens, d_model, generator=gen, device="cuda").to(torch.bfloat16)
    positions = torch.arange(tokens, device="cuda") + 1000
    ids = torch.rand(tokens, vocab, generator=gen, device="cuda").topk(top).indices
    teacher = 2 * torch.randn(tokens, top, generator=gen, device="cuda")
    weight = torch.full((tokens,), 1.0 / tokens, device="cuda")
    weight[7::8] = 0.0                                  # padding
    got = layer.step(x, positions, ids, teacher, weight, temperature)
    want = layer.plain_step(x, positions, ids, teacher, weight, temperature)
    off = lambda g, w, terms: float((g.float() - w).norm() / terms.norm())
    errors = {name: off(g, w, w) for name, g, w in zip(("loss", "dx"), got, want)}
    for name, g, terms in zip(("dw_q", "dw_k"), got[2:], want[2:]):
        errors[name] = off(g, terms.sum((0, 1)), terms)
    if lordba.device_status() != 0:
        raise RuntimeError("a device-side wait ran out")
    return errors


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--d-model", type=int, default=4096)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--top", type=int, default=64)
    ap.add_argument("--rank", type=int, default=16)
    a = ap.parse_args()
    for name, e in run(a.tokens, a.d_model, a.d_model // 128, max(1, a.d_model // 512), 128, a.vocab, a.top, a.rank).items():
        print("%-5s relative error %.2e" % (name, e))
