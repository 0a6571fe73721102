"""Cases of the operators that stand next to the adapters: the frozen base projection in 8-bit integers,
the gated feed-forward block with its backward pass, and dropout from a counter-based generator.

``run`` makes ONE pass through an operator: in plain torch (``own`` false: elementary operations in
32 bits, one rounding at the end) or through the library's calls (``own`` true).  ``exact`` gives the
same outputs from the definitions in 64 bits.
"""
import math

import torch

own = False

DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}

# The most work of one pass: a 8192-token prompt through an 11008 x 4096 projection.
MOST_FLOPS = 2.0 * 8192 * 11008 * 4096
MOST_ELEMENTS = 8192 * 11008


def listed():
    """The sizes are those of the seven adapted projections (4096 -> 4096, 4096 -> 11008, 11008 -> 4096) at
    the token counts at which the adapters are used and measured, and odd ones."""
    return [
        # one new token of one sequence through the gate projection of a quantised base: all latency and weight bytes
        dict(name="int8 one token", op="int8", quantise=True, T=1, d_in=4096, d_out=11008, dtype="bf16", pad=0),
        # a prompt through an attention projection: the activations are quantised on the way
        dict(name="int8 prompt", op="int8", quantise=True, T=2048, d_in=4096, d_out=4096, dtype="bf16", pad=0),
        # a long batch through the down projection, activations quantised before (they serve several projections)
        dict(name="int8 long batch", op="int8", quantise=False, T=8192, d_in=11008, d_out=4096, dtype="f16", pad=0),
        # a small model with widths that nothing divides, float32 outputs
        dict(name="int8 ragged", op="int8", quantise=False, T=777, d_in=1001, d_out=1533, dtype="f32", pad=0),
        # eight sequences that decode together through gate and up
        dict(name="gated decode", op="gated", bits=16, T=8, d_in=4096, d_hidden=11008, dtype="bf16", act="silu", adapters=False, save=False, pad=0),
        # the forward pass of a fine-tuning step: adapters' terms added, pre-activations kept for the backward pass
        dict(name="gated training", op="gated", bits=16, T=2048, d_in=4096, d_hidden=11008, dtype="bf16", act="silu", adapters=True, save=True, pad=0),
        # a prompt through gate and up of a quantised base
        dict(name="gated int8 prompt", op="gated", bits=8, T=1024, d_in=4096, d_hidden=11008, dtype="bf16", act="silu", adapters=False, save=False, pad=0),
        # the backward pass of a fine-tuning step in which the weights learn too
        dict(name="gated gradients", op="gated_grad", T=2048, d_in=4096, d_hidden=11008, dtype="bf16", act="silu", weights=True, pad=0),
        # adapters alone learn (frozen weights): a short ragged batch, the other activation, widths that nothing divides
        dict(name="gated gradients ragged", op="gated_grad", T=333, d_in=520, d_hidden=1365, dtype="f16", act="gelu_tanh", weights=False, pad=0),
        # dropout in front of an adapter in a fine-tuning step
        dict(name="dropout training", op="dropout", T=2048, d=4096, dtype="bf16", p=0.05, residual=False, pad=0),
        # a handful of rows, not a multiple of anything, joined to the residual stream
        dict(name="dropout small", op="dropout", T=7, d=1021, dtype="f32", p=0.1, residual=True, pad=3),
        # a long batch at the hidden width, joined to the residual stream
        dict(name="dropout large", op="dropout", T=8192, d=11008, dtype="bf16", p=0.1, residual=True, pad=0),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, low, high):
    """A width over the logarithm of its range: half of them multiples of 64 (what models have), half anything."""
    d = _log(rng, low, high)
    if rng.random() < 0.5:
        d = max(low, d // 64 * 64)
    return d + 1 if d == 3072 else d


def _tokens(rng, high, flops_per_token):
    return max(1, min(_log(rng, 1, high), int(MOST_FLOPS / flops_per_token)))


def draw(rng):
    op = rng.choice(["int8", "gated", "gated_grad", "dropout"])
    pad = rng.choice([0, 0, 8, 64, 5])      # columns between the end of a row and the next one
    half = rng.choice(["bf16", "f16"])
    act = rng.choice(["silu", "silu", "gelu_tanh"])
    if op == "int8":
        d_in, d_out = _width(rng, 64, 11008), _width(rng, 64, 11008)
        return dict(op=op, quantise=rng.random() < 0.5, T=_tokens(rng, 8192, 2.0 * d_in * d_out), d_in=d_in, d_out=d_out,
                    dtype=rng.choice(["bf16", "f16"]) if rng.random() < 0.8 else "f32", pad=pad)
    if op == "dropout":
        d = _width(rng, 64, 11008)
        return dict(op=op, T=max(1, min(_log(rng, 1, 16384), MOST_ELEMENTS // (d + pad))), d=d, dtype=rng.choice(["bf16", "f16", "f32"]),
                    p=rng.choice([0.0, 0.05, 0.1, 0.3, 0.5]), residual=rng.random() < 0.5, pad=pad)
    d_in, d_hidden = _width(rng, 64, 4096), _width(rng, 64, 11008)
    if op == "gated":
        return dict(op=op, bits=rng.choice([16, 16, 8]), T=_tokens(rng, 8192, 4.0 * d_in * d_hidden), d_in=d_in, d_hidden=d_hidden, dtype=half,
                    act=act, adapters=rng.random() < 0.5, save=rng.random() < 0.5, pad=pad)
    return dict(op=op, T=_tokens(rng, 8192, 8.0 * d_in * d_hidden), d_in=d_in, d_hidden=d_hidden, dtype=half, act=act,
                weights=rng.random() < 0.5, pad=pad)


# ------------------------------------------------------------------------------------------- inputs


def _matrix(gen, rows, cols, dtype, pad=0, scale=1.0):
    """rows x cols of N(0, scale), as a view of a wider buffer where rows are padded."""
    buf = torch.randn(rows, cols + pad, generator=gen, device=DEVICE, dtype=torch.float32)
    return buf.mul_(scale).to(dtype)[:, :cols]


def _activations(gen, rows, cols, dtype, pad=0):
    """N(0, 1) with one channel in a hundred twenty times as large, as trained models have them; one row in
    64 is padding (zero)."""
    x = torch.randn(rows, cols + pad, generator=gen, device=DEVICE, dtype=torch.float32)
    loud = torch.rand(cols + pad, generator=gen, device=DEVICE) < 0.01
    x.mul_(torch.where(loud, 20.0, 1.0))
    x[63::64] = 0.0
    return x.to(dtype)[:, :cols]


def _int8(gen, rows, cols, pad=0):
    """rows x cols integers of -127 ... 127, spread as quantised Gaussians are."""
    q = torch.randn(rows, cols + pad, generator=gen, device=DEVICE, dtype=torch.float32)
    return q.mul_(32.0).round_().clamp_(-127, 127).to(torch.int8)[:, :cols]


def _scales(gen, n, typical):
    """Positive scales, log-normal around a typical value."""
    return torch.randn(n, generator=gen, device=DEVICE, dtype=torch.float32).mul_(0.5).exp_().mul_(typical)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    s = dict(case)
    dtype = TYPES[case["dtype"]]
    T, pad, op = case["T"], case["pad"], case["op"]
    if op == "dropout":
        s["x"] = _matrix(gen, T, case["d"], dtype, pad)
        s["r"] = _matrix(gen, T, case["d"], dtype, pad) if case["residual"] else None
        s["seed"], s["offset"] = 0x9E3779B97F4A7C15 ^ int(seed), 1000 + int(seed)
        return s
    d_in = case["d_in"]
    n = case["d_out"] if op == "int8" else case["d_hidden"]
    if op == "int8":
        s["w"], s["s_w"] = _int8(gen, n, d_in, pad), _scales(gen, n, 1 / (32.0 * math.sqrt(d_in)))
        if case["quantise"]:
            s["x"] = _activations(gen, T, d_in, dtype, pad)
        else:
            s["x"], s["s_x"] = _int8(gen, T, d_in, pad), _scales(gen, T, 1 / 32.0)
        return s
    if op == "gated" and case["bits"] == 8:
        s["x"], s["s_x"] = _int8(gen, T, d_in, pad), _scales(gen, T, 1 / 32.0)
        s["w_gate"], s["s_gate"] = _int8(gen, n, d_in, pad), _scales(gen, n, 1 / (32.0 * math.sqrt(d_in)))
        s["w_up"], s["s_up"] = _int8(gen, n, d_in, pad), _scales(gen, n, 1 / (32.0 * math.sqrt(d_in)))
    else:
        s["x"] = _matrix(gen, T, d_in, dtype, pad)
        s["w_gate"] = _matrix(gen, n, d_in, dtype, pad, 1 / math.sqrt(d_in))
        s["w_up"] = _matrix(gen, n, d_in, dtype, pad, 1 / math.sqrt(d_in))
    if op == "gated":
        s["g0"] = _matrix(gen, T, n, dtype, pad, 0.25) if case["adapters"] else None
        s["u0"] = _matrix(gen, T, n, dtype, pad, 0.25) if case["adapters"] else None
    else:
        s["gate"], s["up"], s["dh"] = (_matrix(gen, T, n, dtype, pad) for _ in range(3))
    return s


# ------------------------------------------------------------------------------------ the plain form


def _plain_quantise(x):
    """A scale for each row, amax / 127, and the integers that x / scale rounds to (ties to even)."""
    x = x.float()
    amax = x.abs().amax(dim=1, keepdim=True)
    inverse = torch.where(amax > 0, torch.full_like(amax, 127.0) / amax, torch.zeros_like(amax))
    return torch.round(x * inverse), amax / 127.0


def _plain_int8(x, s_x, w, s_w):
    return (x.float() @ w.float().T) * s_x.reshape(-1, 1) * s_w


def _sigmoid_of(g, act):
    """The factor f of act(g) = g f(g), and the argument's derivative."""
    if act == "silu":
        return torch.sigmoid(g), 1.0
    k = 2.0 * math.sqrt(2.0 / math.pi)
    return torch.sigmoid(k * (g + 0.044715 * g * g * g)), k * (1.0 + 3 * 0.044715 * g * g)


def _plain_gated(s):
    dtype = TYPES[s["dtype"]]
    if s["bits"] == 8:
        g, u = _plain_int8(s["x"], s["s_x"], s["w_gate"], s["s_gate"]), _plain_int8(s["x"], s["s_x"], s["w_up"], s["s_up"])
    else:
        g, u = s["x"].float() @ s["w_gate"].float().T, s["x"].float() @ s["w_up"].float().T
    if s["adapters"]:
        g, u = g + s["g0"].float(), u + s["u0"].float()
    f, _ = _sigmoid_of(g, s["act"])
    out = {"h": (g * f * u).to(dtype)}
    if s["save"]:
        out["gate"], out["up"] = g.to(dtype), u.to(dtype)
    return out


def _plain_gated_grad(s):
    dtype = TYPES[s["dtype"]]
    g, u, dh = s["gate"].float(), s["up"].float(), s["dh"].float()
    f, inner = _sigmoid_of(g, s["act"])
    dg, du = dh * u * f * (1.0 + g * (1.0 - f) * inner), dh * g * f
    out = {"dgate": dg.to(dtype), "dup": du.to(dtype), "dx": (dg @ s["w_gate"].float() + du @ s["w_up"].float()).to(dtype)}
    if s["weights"]:
        x = s["x"].float()
        out["dw_gate"], out["dw_up"] = (dg.T @ x).to(dtype), (du.T @ x).to(dtype)
    return out


def _plain_bits(T, d, seed, offset, device):
    """The 16-bit numbers of a T x d matrix: eight from each block of Philox4x32-10 (Salmon et al. 2011), whose
    counter is (column / 8, row, offset) and whose key is the seed."""
    low = 0xFFFFFFFF
    groups = (d + 7) // 8
    zero = torch.zeros(T, groups, dtype=torch.int64, device=device)
    c0 = zero + torch.arange(groups, device=device)
    c1 = zero + torch.arange(T, device=device).reshape(-1, 1)
    c2, c3 = zero + (offset & low), zero + (offset >> 32 & low)
    k0, k1 = seed & low, seed >> 32 & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (b >> 32 & low) ^ c1 ^ k0, b & low, (a >> 32 & low) ^ c3 ^ k1, a & low
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    words = torch.stack([c0, c1, c2, c3], dim=2)
    return torch.stack([words & 0xFFFF, words >> 16], dim=3).reshape(T, groups * 8)[:, :d]


def _plain_dropout(s):
    x = s["x"].float()
    cut = int(round(s["p"] * 65536))
    keep = _plain_bits(s["T"], s["d"], s["seed"], s["offset"], x.device) >= cut
    y = torch.where(keep, x * (65536.0 / (65536 - cut)), torch.zeros_like(x))
    if s["r"] is not None:
        y = y + s["r"].float()
    return y.to(TYPES[s["dtype"]])


def _run_plain(s):
    if s["op"] == "int8":
        x, s_x = _plain_quantise(s["x"]) if s["quantise"] else (s["x"], s["s_x"])
        return _plain_int8(x, s_x, s["w"], s["s_w"]).to(TYPES[s["dtype"]])
    return {"gated": _plain_gated, "gated_grad": _plain_gated_grad, "dropout": _plain_dropout}[s["op"]](s)


# --------------------------------------------------------------------------------- the library's calls


def _run_own(s):
    from paper_2605_24058_b200 import lordba
    op, dtype = s["op"], TYPES[s["dtype"]]
    if op == "dropout":
        return lordba.dropout(s["x"], s["p"], s["seed"], s["offset"], residual=s["r"])
    if op == "int8":
        x, s_x = lordba.int8_quantize_rows(s["x"]) if s["quantise"] else (s["x"], s["s_x"])
        return lordba.int8_linear(x, s_x, s["w"], s["s_w"], dtype=dtype)
    act = lordba.ACT_SILU if s["act"] == "silu" else lordba.ACT_GELU_TANH
    if op == "gated":
        scales = (s["s_x"], s["s_gate"], s["s_up"]) if s["bits"] == 8 else None
        h, gate, up = lordba.gated_forward(s["x"], s["w_gate"], s["w_up"], act=act, scales=scales, dtype=dtype,
                                           gate_add=s["g0"], up_add=s["u0"], save=s["save"])
        return {"h": h, "gate": gate, "up": up} if s["save"] else {"h": h}
    got = lordba.gated_backward(s["dh"], s["gate"], s["up"], s["x"] if s["weights"] else None, s["w_gate"], s["w_up"], act=act)
    names = ("dgate", "dup", "dx", "dw_gate", "dw_up") if s["weights"] else ("dgate", "dup", "dx")
    return dict(zip(names, got))


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------ the work


def work(case):
    T, e, op = case["T"], SIZE[case["dtype"]], case["op"]
    if op == "dropout":
        n = T * case["d"]
        return {"bytes": n * e * (3 if case["residual"] else 2), "flops": 2 * n}
    d = case["d_in"]
    if op == "int8":
        n = case["d_out"]
        x = T * d * e if case["quantise"] else T * d + 4 * T
        return {"bytes": x + n * d + 4 * n + T * n * e, "flops": 2 * T * d * n}
    n = case["d_hidden"]
    if op == "gated":
        inputs = T * d + 4 * T + 2 * n * (d + 4) if case["bits"] == 8 else (T * d + 2 * n * d) * e
        return {"bytes": inputs + T * n * e * (1 + 2 * case["adapters"] + 2 * case["save"]), "flops": 4 * T * d * n}
    both = 1 + case["weights"]
    return {"bytes": (5 * T * n + both * (T * d + 2 * n * d)) * e, "flops": both * 4 * T * d * n}


# --------------------------------------------------------------------------- the definitions in 64 bits


def _exact_product(x, s_x, w, s_w):
    """Integer sums are exact in 64-bit floats (below 2^53); then one scale a row, one a column."""
    return torch.einsum("tk,nk->tn", x.double(), w.double()) * torch.outer(s_x.double().reshape(-1), s_w.double())


def _exact_act(g, act):
    """Value and derivative of the activation."""
    if act == "silu":
        e = torch.exp(-g)
        return g / (1 + e), (1 + e + g * e) / (1 + e) ** 2
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return g * (1 + t) / 2, (1 + t) / 2 + g * (1 - t ** 2) / 2 * c * (1 + 0.134145 * g ** 2)


def _exact_mul(a, m):
    """High and low word of a product of two 32-bit numbers, by 16-bit halves."""
    lo, hi = (a % 65536) * m, (a // 65536) * m
    total = lo // 65536 + hi
    return total // 65536, (total % 65536) * 65536 + lo % 65536


def _exact_keep(first, T, d, seed, offset, cut):
    """Which elements of rows first ... first + T - 1 stay."""
    two32 = 1 << 32
    col = torch.arange(d, device=DEVICE)
    row = torch.arange(first, first + T, device=DEVICE)
    c = [(col // 8).expand(T, d), row.reshape(T, 1).expand(T, d), torch.full((T, d), offset % two32, device=DEVICE),
         torch.full((T, d), offset // two32 % two32, device=DEVICE)]
    for i in range(10):
        key = (seed + i * 0x9E3779B9) % two32, (seed // two32 + i * 0xBB67AE85) % two32
        h0, l0 = _exact_mul(c[0], 0xD2511F53)
        h1, l1 = _exact_mul(c[2], 0xCD9E8D57)
        c = [h1 ^ c[1] ^ key[0], l1, h0 ^ c[3] ^ key[1], l0]
    word = torch.stack(c)[(col % 8 // 2).expand(1, T, d), (row - first).reshape(1, T, 1), col.reshape(1, 1, d)][0]
    return torch.where(col % 2 == 1, word // 65536, word % 65536) >= cut


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "dropout":
        cut = int(round(case["p"] * 65536))
        y = s["x"].double() * 65536 / (65536 - cut)
        step = max(1, (1 << 23) // case["d"])            # rows at a time: the counters are eight bytes each
        for i in range(0, case["T"], step):
            part = y[i:i + step]
            part[~_exact_keep(i, part.shape[0], case["d"], s["seed"], s["offset"], cut)] = 0
        return y if s["r"] is None else y + s["r"].double()
    if op == "int8":
        x, s_x = s["x"], s.get("s_x")
        if case["quantise"]:
            s_x = x.double().abs().amax(1) / 127
            x = torch.round(x.double() / torch.where(s_x > 0, s_x, torch.ones_like(s_x)).reshape(-1, 1))
        return _exact_product(x, s_x, s["w"], s["s_w"])
    if op == "gated":
        if case["bits"] == 8:
            g, u = (_exact_product(s["x"], s["s_x"], s["w_" + k], s["s_" + k]) for k in ("gate", "up"))
        else:
            g, u = (torch.einsum("td,nd->tn", s["x"].double(), s["w_" + k].double()) for k in ("gate", "up"))
        if case["adapters"]:
            g, u = g + s["g0"].double(), u + s["u0"].double()
        out = {"h": _exact_act(g, case["act"])[0] * u}
        return {**out, "gate": g, "up": u} if case["save"] else out
    dh, u = s["dh"].double(), s["up"].double()
    value, slope = _exact_act(s["gate"].double(), case["act"])
    dg, du = dh * u * slope, dh * value
    out = {"dgate": dg, "dup": du,
           "dx": torch.einsum("tn,nd->td", dg, s["w_gate"].double()) + torch.einsum("tn,nd->td", du, s["w_up"].double())}
    if case["weights"]:
        x = s["x"].double()
        out["dw_gate"], out["dw_up"] = torch.einsum("tn,td->nd", dg, x), torch.einsum("tn,td->nd", du, x)
    return out
