"""An adapted feed-forward block, served over an 8-bit base and fine-tuned over a 16-bit one.

The block is  h = silu(g) * u,  y = W_down h  with  g = W_gate x + adapter_gate(x),  u = W_up x + adapter_up(x)
and the down projection adapted as well.  Serving quantises the activations per token on the way into each base
projection; a training step drops out the adapters' inputs, keeps g and u, and brings the gradient of y back to
the block's input (the base weights stay frozen, their gradients can be asked for).

    python examples/adapted_feed_forward.py [--tokens T] [--d-model D] [--d-hidden F] [--rank R]

prints how far both are from the same block in plain float32 torch.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_24058_b200 import lordba  # noqa: E402


class Adapter:
    """A double-binary adapter d_in -> d_out of rank r, and its adjoint (the same call with swapped roles)."""

    def __init__(self, d_in, d_out, r, gen, gain):
        dev = "cuda"
        sign = lambda a, b: torch.randint(0, 2, (a, b), generator=gen, device=dev, dtype=torch.int8) * 2 - 1
        scale = lambda n, m=1.0: torch.randn(n, generator=gen, device=dev).mul_(0.3).exp_() * m
        self.r, self.A, self.B = r, sign(r, d_in), sign(d_out, r)
        self.s_in, self.s_r, self.s_out = scale(d_in), scale(r, gain / (r * d_in) ** 0.5), scale(d_out)
        self.forward_carriers = lordba.pack_signs(self.A, 0), lordba.pack_signs(self.B, 1)
        self.adjoint_carriers = lordba.pack_signs(self.B.t().contiguous(), 0), lordba.pack_signs(self.A.t().contiguous(), 1)

    def add_to(self, x, y):
        lordba.adapter_forward(x, *self.forward_carriers, self.s_in, self.s_r, self.s_out, y, self.r)

    def add_adjoint_to(self, dy, dx):
        lordba.adapter_forward(dy, *self.adjoint_carriers, self.s_out, self.s_r, self.s_in, dx, self.r)

    def dense(self):
        """Delta-W as d_out x d_in, for comparison."""
        return (self.s_out[:, None] * self.B * self.s_r) @ (self.A * self.s_in)


class Block:
    def __init__(self, d_model, d_hidden, rank, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        weight = lambda a, b: (torch.randn(a, b, generator=gen, device="cuda") / b ** 0.5).to(torch.bfloat16)
        self.gate, self.up, self.down = weight(d_hidden, d_model), weight(d_hidden, d_model), weight(d_model, d_hidden)
        # once: the base in 8 bits, one scale an output channel
        self.base8 = [lordba.int8_quantize_rows(w) for w in (self.gate, self.up, self.down)]
        self.adapters = [Adapter(d_model, d_hidden, rank, gen, 0.5), Adapter(d_model, d_hidden, rank, gen, 0.5),
                         Adapter(d_hidden, d_model, rank, gen, 0.5)]

    def adapter_terms(self, x):
        """What the adapters of gate and up add, in one launch over zeroed buffers."""
        terms = [torch.zeros(x.shape[0], w.shape[0], dtype=x.dtype, device=x.device) for w in (self.gate, self.up)]
        projs = [lordba.make_proj(x, *a.forward_carriers, a.s_in, a.s_r, a.s_out, t, a.r) for a, t in zip(self.adapters, terms)]
        lordba.adapter_forward_batched(projs, x.shape[0], lordba.BF16)
        return terms

    def serve(self, x):
        (gate8, s_gate), (up8, s_up), (down8, s_down) = self.base8
        x8, s_x = lordba.int8_quantize_rows(x)
        g0, u0 = self.adapter_terms(x)
        h, _, _ = lordba.gated_forward(x8, gate8, up8, scales=(s_x, s_gate, s_up), gate_add=g0, up_add=u0, dtype=x.dtype)
        h8, s_h = lordba.int8_quantize_rows(h)
        y = lordba.int8_linear(h8, s_h, down8, s_down, dtype=x.dtype)
        self.adapters[2].add_to(h, y)
        return y

    def forward(self, x, p, seed, step):
        """y and what the backward pass needs.  The adapters' inputs are dropped out; no mask is kept."""
        dropped = lordba.dropout(x, p, seed, 2 * step)
        g0, u0 = self.adapter_terms(dropped)
        h, gate, up = lordba.gated_forward(x, self.gate, self.up, gate_add=g0, up_add=u0, save=True)
        y = h @ self.down.t()
        self.adapters[2].add_to(lordba.dropout(h, p, seed, 2 * step + 1), y)
        return y, (gate, up)

    def backward(self, dy, saved, p, seed, step, x=None):
        """(gradient of x, of g, of u, of W_gate and W_up or None): the last two where x is given."""
        gate, up = saved
        dropped = torch.zeros(dy.shape[0], self.gate.shape[0], dtype=dy.dtype, device=dy.device)
        self.adapters[2].add_adjoint_to(dy, dropped)
        dh = lordba.dropout(dropped, p, seed, 2 * step + 1, residual=dy @ self.down)
        dgate, dup, dx, dw_gate, dw_up = lordba.gated_backward(dh, gate, up, x, self.gate, self.up)
        dropped = torch.zeros_like(dx)
        self.adapters[0].add_adjoint_to(dgate, dropped)
        self.adapters[1].add_adjoint_to(dup, dropped)
        dx = lordba.dropout(dropped, p, seed, 2 * step, residual=dx)
        return dx, dgate, dup, dw_gate, dw_up

    # ---- the same in plain float32 torch ----------------------------------------------------------------------
    def plain_serve(self, x):
        w = [q.float() * s[:, None] for q, s in self.base8]
        d = [a.dense() for a in self.adapters]

        def through(v, k):
            s = v.abs().amax(1, keepdim=True) / 127
            return torch.round(v / torch.where(s > 0, s, torch.ones_like(s))) * s @ w[k].t()

        x = x.float()
        g, u = through(x, 0) + x @ d[0].t(), through(x, 1) + x @ d[1].t()
        h = torch.sigmoid(g) * g * u
        return through(h, 2) + h @ d[2].t()

    def plain_step(self, x, dy, p, seed, step):
        """y, dx, dW_gate, dW_up by torch's own differentiation, with the masks that dropout() draws."""
        w = [v.float().requires_grad_(k < 2) for k, v in enumerate((self.gate, self.up, self.down))]
        d = [a.dense() for a in self.adapters]
        mask = lambda like, offset: lordba.dropout(torch.ones_like(like, dtype=torch.float32), p, seed, offset)
        x = x.float().requires_grad_(True)
        xd = x * mask(x, 2 * step)
        g, u = x @ w[0].t() + xd @ d[0].t(), x @ w[1].t() + xd @ d[1].t()
        h = torch.sigmoid(g) * g * u
        y = h @ w[2].t() + (h * mask(h, 2 * step + 1)) @ d[2].t()
        y.backward(dy.float())
        return y.detach(), x.grad, w[0].grad, w[1].grad


def run(tokens, d_model, d_hidden, rank, p=0.1, seed=1):
    """Relative errors (2-norm) of the served output and of a training step's output and gradients."""
    block = Block(d_model, d_hidden, rank, seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 1)
    x, dy = (torch.randn(tokens, d_model, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    off = lambda got, want: float((got.float() - want).norm() / want.norm())
    errors = {"served": off(block.serve(x), block.plain_serve(x))}
    y, saved = block.forward(x, p, seed, 3)
    dx, _, _, dw_gate, dw_up = block.backward(dy, saved, p, seed, 3, x)
    want = block.plain_step(x, dy, p, seed, 3)
    for name, got, ref in zip(("output", "dx", "dw_gate", "dw_up"), (y, dx, dw_gate, dw_up), want):
        errors[name] = off(got, ref)
    if lordba.device_status() != 0:
        raise RuntimeError("a device-side wait ran out")
    return errors


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--d-model", type=int, default=4096)
    ap.add_argument("--d-hidden", type=int, default=11008)
    ap.add_argument("--rank", type=int, default=16)
    a = ap.parse_args()
    for name, e in run(a.tokens, a.d_model, a.d_hidden, a.rank).items():
        print("%-8s relative error %.2e" % (name, e))
