"""Cases of the operators for an adapter that is trained and served over a 4-bit base: products with 4-bit weights
and group scales (and their gradient to the activations), norms of queries and keys with the position rotation (and
their gradients), and distillation from a teacher's top logits (loss and gradient).

``run`` makes ONE pass through an operator: in plain torch (``own`` false: elementary operations in 32 bits, angles in
64, one rounding at the end) or through the library's calls (``own`` true).  ``exact`` gives the same outputs from the
definitions in 64 bits.
"""
import math

import torch

own = False

DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}

# The most work of one pass, of each operator: that of its largest listed case.
MOST_FLOPS = 2.0 * 2048 * 11008 * 4096
MOST_HEADS = 8192 * 40 * 128
MOST_LOGITS = 4096 * 131072


def listed():
    """Projections of 4096 and 11008 wide activations, 32 heads of 128, a vocabulary of 32000: the shapes whose adapters
    this repository measures; and generic ones."""
    return [
        # one new token of one sequence through the gate projection of a 4-bit base: all latency and weight bytes
        dict(name="int4 one token", op="int4", T=1, d_in=4096, d_out=11008, group=128, zeros=False, dtype="bf16", pad=0),
        # sixteen sequences that decode together through the down projection; a checkpoint with zero points
        dict(name="int4 decode", op="int4", T=16, d_in=11008, d_out=4096, group=64, zeros=True, dtype="f16", pad=0),
        # a short prompt through an attention projection
        dict(name="int4 short prompt", op="int4", T=56, d_in=4096, d_out=4096, group=128, zeros=False, dtype="bf16", pad=0),
        # a training batch, or a long prompt, through the gate projection
        dict(name="int4 prompt", op="int4", T=2048, d_in=4096, d_out=11008, group=128, zeros=False, dtype="bf16", pad=0),
        # the same batch on the way back: the gradient that the frozen projection hands down
        dict(name="int4 gradient", op="int4_grad", T=2048, d_in=4096, d_out=11008, group=128, zeros=False, dtype="bf16", pad=0),
        # a small model with widths that nothing divides, rows off the 16-byte grid
        dict(name="int4 gradient ragged", op="int4_grad", T=333, d_in=1001, d_out=1533, group=32, zeros=True, dtype="f16", pad=5),
        # one new token, rotation alone: all latency
        dict(name="rotation one token", op="rope", T=1, heads_q=32, heads_k=32, d=128, rotary=128, norm=False, interleaved=False, dtype="bf16", pad=0),
        # a long prompt, shared key heads, queries and keys as they lie in one joint projection's output
        dict(name="norm and rotation prompt", op="rope", T=8192, heads_q=32, heads_k=8, d=128, rotary=128, norm=True, interleaved=False, dtype="bf16", pad=1024),
        # the way back in a training step, the norms' weights learn
        dict(name="norm and rotation gradients", op="rope_grad", T=4096, heads_q=32, heads_k=8, d=128, rotary=128, norm=True, interleaved=False, dtype="bf16", pad=0),
        # a training step's loss and its gradient in one call: the weights of the rows are known
        dict(name="distillation step", op="distill", mode="step", T=2048, V=32000, top=64, tau=2.0, dtype="bf16", pad=0),
        # a large batch over a large vocabulary
        dict(name="distillation large", op="distill", mode="step", T=4096, V=131072, top=32, tau=1.0, dtype="bf16", pad=0),
        # the loss alone, of a handful of tokens in 32 bits, a width that nothing divides
        dict(name="distillation loss", op="distill", mode="loss", T=7, V=32003, top=20, tau=1.0, dtype="f32", pad=1),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, low, high):
    """A width over the logarithm of its range: half of them multiples of 64 (what models have), half anything."""
    d = _log(rng, low, high)
    return max(low, d // 64 * 64) if rng.random() < 0.5 else d


def draw(rng):
    op = rng.choice(["int4", "int4", "int4_grad", "rope", "rope_grad", "distill", "distill"])
    pad = rng.choice([0, 0, 8, 64, 5])      # columns between the end of a row and the next one
    if op in ("int4", "int4_grad"):
        d_in, d_out = _width(rng, 64, 11008), _width(rng, 64, 11008)
        T = max(1, min(_log(rng, 1, 4096), int(MOST_FLOPS / (2.0 * d_in * d_out))))
        return dict(op=op, T=T, d_in=d_in, d_out=d_out, group=rng.choice([32, 64, 128, 128]), zeros=rng.random() < 0.5,
                    dtype=rng.choice(["bf16", "f16"]), pad=pad)
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("rope", "rope_grad"):
        d = rng.choice([64, 64, 128, 128, 128, 256, 80, 96, 2 * rng.randint(4, 128)])
        heads_k = rng.choice([1, 2, 4, 8, rng.randint(1, 12)])
        heads_q = heads_k * rng.choice([1, 2, 4, 8])
        T = max(1, min(_log(rng, 1, 16384), MOST_HEADS // ((heads_q + heads_k) * d)))
        return dict(op=op, T=T, heads_q=heads_q, heads_k=heads_k, d=d, rotary=rng.choice([d, d, d, max(2, d // 4 * 2)]),
                    norm=rng.random() < 0.75, interleaved=rng.random() < 0.3, dtype=dtype, pad=pad)
    V = _width(rng, 1000, 160000)
    T = max(1, min(_log(rng, 1, 8192), MOST_LOGITS // (V * SIZE[dtype] // 2)))
    return dict(op=op, mode=rng.choice(["step", "step", "loss", "backward"]), T=T, V=V, top=_log(rng, 1, 128), tau=rng.choice([1.0, 1.0, 2.0, 4.0, 0.7]),
                dtype=dtype, pad=pad)


# ------------------------------------------------------------------------------------------- inputs


def _matrix(gen, rows, cols, dtype, pad=0, scale=1.0):
    """rows x cols of N(0, scale), as a view of a wider buffer where rows are padded."""
    buf = torch.randn(rows, cols + pad, generator=gen, device=DEVICE, dtype=torch.float32)
    return buf.mul_(scale).to(dtype)[:, :cols]


def _pack(u):
    """4-bit values (d_out, d_in) as the library's carrier: blocks of 128 columns, 64 bytes of sixteen 32-bit words.  Word
    4 t + j holds columns 32 j + 8 t ... + 7 of the block, column c of these in bits 4 (c / 2) + 16 (c % 2) on."""
    rows, cols = u.shape
    blocks = (cols + 127) // 128
    full = torch.zeros(rows, blocks * 128, dtype=torch.int64, device=u.device)
    full[:, :cols] = u
    shift = torch.tensor([4 * (c // 2) + 16 * (c % 2) for c in range(8)], device=u.device)
    words = (full.reshape(rows, blocks, 4, 4, 8) << shift).sum(-1)            # [row, block, j, t]
    words = words.permute(0, 1, 3, 2).reshape(rows, blocks * 16)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32).view(torch.uint8)


def _positions(gen, T):
    """One token each of many sequences, or sequences of up to 2048 tokens one after the other, each from its own start."""
    if T <= 64:
        return torch.randint(0, 131072, (T,), generator=gen, device=DEVICE)
    at = torch.arange(T, device=DEVICE)
    start = torch.randint(0, 100000, (T // 2048 + 1,), generator=gen, device=DEVICE)
    return start[at // 2048] + at % 2048


def _logits(s, case, gen):
    """Student's logits, the teacher's top ones (some rows have fewer than the rest), and the rows' weights: one row in
    sixteen is padding."""
    T, V, top, dtype = case["T"], case["V"], case["top"], TYPES[case["dtype"]]
    buf = torch.empty(T, V + case["pad"], dtype=dtype, device=DEVICE)
    ids = torch.empty(T, top, dtype=torch.int64, device=DEVICE)
    values = torch.empty(T, top, dtype=torch.float32, device=DEVICE)
    step = max(1, (1 << 27) // V)
    for i in range(0, T, step):
        n = min(step, T - i)
        teacher = torch.randn(n, V, generator=gen, device=DEVICE).mul_(2.5)
        values[i:i + n], ids[i:i + n] = torch.topk(teacher, top, dim=1)
        buf[i:i + n, :V] = teacher.add_(torch.randn(n, V, generator=gen, device=DEVICE), alpha=0.5).to(dtype)
    if V + case["pad"] > V:
        buf[:, V:] = 0
    fewer = torch.randint(1, top + 1, (T, 1), generator=gen, device=DEVICE)
    absent = (torch.arange(top, device=DEVICE) >= fewer) & (torch.arange(T, device=DEVICE) % 5 == 3).reshape(-1, 1)
    s["logits"], s["ids"], s["teacher"] = buf[:, :V], torch.where(absent, torch.full_like(ids, -1), ids), values.to(dtype)
    padding = torch.arange(T, device=DEVICE) % 16 == 15
    s["weight"] = torch.where(padding, 0.0, 1.0 / T).float()
    if case["mode"] == "backward":
        lse = torch.empty(T, dtype=torch.float32, device=DEVICE)
        for i in range(0, T, step):
            lse[i:i + step] = torch.logsumexp(s["logits"][i:i + step].double() / case["tau"], 1).float()
        s["lse"] = lse


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    s = dict(case)
    T, pad, dtype, op = case["T"], case["pad"], TYPES[case["dtype"]], case["op"]
    if op in ("int4", "int4_grad"):
        d_in, n, groups = case["d_in"], case["d_out"], -(-case["d_in"] // case["group"])
        u = torch.randn(n, d_in, generator=gen, device=DEVICE).mul_(3.0).round_().clamp_(-8, 7).to(torch.int64).add_(8)
        s["q"] = _pack(u)
        s["scale"] = torch.randn(n, groups, generator=gen, device=DEVICE).mul_(0.3).exp_().mul_(1 / (3.0 * math.sqrt(d_in))).to(dtype)
        s["zero"] = torch.randint(5, 12, (n, groups), generator=gen, device=DEVICE).to(torch.uint8) if case["zeros"] else None
        s["x" if op == "int4" else "dy"] = _matrix(gen, T, d_in if op == "int4" else n, dtype, pad)
        return s
    if op in ("rope", "rope_grad"):
        d, hq, hk = case["d"], case["heads_q"], case["heads_k"]

        def joint():
            both = _matrix(gen, T, (hq + hk) * d, dtype, pad, 1.5)        # queries and keys of a token in one row
            return both[:, :hq * d].unflatten(1, (hq, d)), both[:, hq * d:].unflatten(1, (hk, d))

        s["q"], s["k"] = joint()
        if op == "rope_grad":
            s["dq_out"], s["dk_out"] = joint()
        s["positions"] = _positions(gen, T)
        s["inv_freq"] = 1.0 / 10000.0 ** (torch.arange(0, case["rotary"], 2, device=DEVICE).float() / case["rotary"])
        learned = lambda: torch.randn(d, generator=gen, device=DEVICE).mul_(0.2).add_(1.0).to(dtype) if case["norm"] else None
        s["w_q"], s["w_k"], s["eps"] = learned(), learned(), 1e-6
        return s
    _logits(s, case, gen)
    return s


# ------------------------------------------------------------------------------------ the plain form


def _plain_weights(s):
    """The matrix (d_out, d_in) in 32 bits."""
    rows = s["q"].shape[0]
    words = s["q"].view(torch.int32).reshape(rows, -1, 4, 4).permute(0, 1, 3, 2)       # [row, block, j, t]
    shift = torch.tensor([4 * (c // 2) + 16 * (c % 2) for c in range(8)], dtype=torch.int32, device=words.device)
    u = ((words.unsqueeze(-1) >> shift) & 15).reshape(rows, -1)[:, :s["d_in"]].float()
    group = torch.arange(s["d_in"], device=u.device) // s["group"]
    zero = s["zero"].float()[:, group] if s["zero"] is not None else 8.0
    return (u - zero) * s["scale"].float()[:, group]


def _plain_int4(s):
    w = _plain_weights(s)
    return (s["x"].float() @ w.T if s["op"] == "int4" else s["dy"].float() @ w).to(TYPES[s["dtype"]])


def _plain_angles(s):
    angle = s["positions"].double().reshape(-1, 1, 1) * s["inv_freq"].double()
    return torch.cos(angle).float(), torch.sin(angle).float()


def _pairs(s):
    """Columns of the first and of the second entries of the rotated pairs."""
    half = s["rotary"] // 2
    return (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if s["interleaved"] else (slice(0, half), slice(half, 2 * half))


def _plain_rotate(x, cos, sin, s):
    a, b = _pairs(s)
    out = x.clone()
    out[..., a] = x[..., a] * cos - x[..., b] * sin
    out[..., b] = x[..., b] * cos + x[..., a] * sin
    return out


def _plain_rope(s):
    cos, sin = _plain_angles(s)
    out = {}
    for name, w in (("q", s["w_q"]), ("k", s["w_k"])):
        x = s[name].float()
        if s["norm"]:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * w.float()
        out[name] = _plain_rotate(x, cos, sin, s).to(TYPES[s["dtype"]])
    return out


def _plain_rope_grad(s):
    cos, sin = _plain_angles(s)
    out = {}
    for name, w in (("q", s["w_q"]), ("k", s["w_k"])):
        x, g = s[name].float(), _plain_rotate(s["d%s_out" % name].float(), cos, -sin, s)
        if s["norm"]:
            r = torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"])
            unit = x * r
            out["dw_" + name] = (g * unit).sum((0, 1))
            g = g * w.float()
            g = r * (g - unit * (g * unit).mean(-1, keepdim=True))
        out["d" + name] = g.to(TYPES[s["dtype"]])
    return out


def _plain_distill(s):
    tau, V, dtype = s["tau"], s["V"], TYPES[s["dtype"]]
    z = s["logits"].float() / tau
    present = s["ids"] >= 0
    v = torch.where(present, s["teacher"].float() / tau, torch.full_like(s["teacher"], -math.inf, dtype=torch.float32))
    e = torch.exp(v - v.amax(1, keepdim=True))
    total = e.sum(1, keepdim=True)
    p = e / total
    if s["mode"] == "backward":
        lse = s["lse"]
    else:
        top = z.amax(1)
        lse = torch.log(torch.exp(z - top.reshape(-1, 1)).sum(1)) + top
    weight, ids = s["weight"], s["ids"].clamp(min=0)
    out = {}
    if s["mode"] != "backward":
        log_p = v - v.amax(1, keepdim=True) - torch.log(total)
        log_q = torch.gather(z, 1, ids) - lse.reshape(-1, 1)
        out["loss"] = weight * tau * tau * torch.where(p > 0, p * (log_p - log_q), torch.zeros_like(p)).sum(1)
        out["lse"] = lse
    if s["mode"] != "loss":
        dz = torch.exp(z - lse.reshape(-1, 1))
        dz.scatter_add_(1, ids, -p)
        out["dlogits"] = (dz * (weight * tau).reshape(-1, 1)).to(dtype)
    return out


def _run_plain(s):
    return {"int4": _plain_int4, "int4_grad": _plain_int4, "rope": _plain_rope, "rope_grad": _plain_rope_grad, "distill": _plain_distill}[s["op"]](s)


# --------------------------------------------------------------------------------- the library's calls


def _run_own(s):
    from paper_2605_24058_b200 import lordba
    op = s["op"]
    if op == "int4":
        return lordba.int4_linear(s["x"], s["q"], s["scale"], zero=s["zero"], group=s["group"])
    if op == "int4_grad":
        return lordba.int4_linear_backward(s["dy"], s["q"], s["scale"], s["d_in"], zero=s["zero"], group=s["group"])
    if op == "rope":
        q, k = lordba.norm_rope(s["q"], s["k"], s["positions"], s["inv_freq"], s["w_q"], s["w_k"], eps=s["eps"], norm=s["norm"], interleaved=s["interleaved"])
        return {"q": q, "k": k}
    if op == "rope_grad":
        dq, dk, dw_q, dw_k = lordba.norm_rope_backward(s["dq_out"], s["dk_out"], s["q"], s["k"], s["positions"], s["inv_freq"], s["w_q"], s["w_k"],
                                                       eps=s["eps"], norm=s["norm"], interleaved=s["interleaved"])
        return {"dw_q": dw_q, "dq": dq, "dw_k": dw_k, "dk": dk} if s["norm"] else {"dq": dq, "dk": dk}
    if s["mode"] == "backward":
        return {"dlogits": lordba.distill_backward(s["weight"], s["logits"], s["ids"], s["teacher"], s["lse"], temperature=s["tau"])}
    loss, lse, dlogits = lordba.distill_loss(s["logits"], s["ids"], s["teacher"], temperature=s["tau"], weight=s["weight"], grad=s["mode"] == "step")
    return {"loss": loss, "lse": lse, "dlogits": dlogits} if s["mode"] == "step" else {"loss": loss, "lse": lse}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------ the work


def work(case):
    T, e, op = case["T"], SIZE[case["dtype"]], case["op"]
    if op in ("int4", "int4_grad"):
        d, n, groups = case["d_in"], case["d_out"], -(-case["d_in"] // case["group"])
        return {"bytes": n * d // 2 + n * groups * (3 if case["zeros"] else 2) + T * (d + n) * e, "flops": 2 * T * d * n}
    if op in ("rope", "rope_grad"):
        n = T * (case["heads_q"] + case["heads_k"]) * case["d"]
        back = op == "rope_grad"
        return {"bytes": n * e * (3 if back else 2) + 8 * T + 2 * case["rotary"] + (2 * case["d"] * (e + 4 * back) if case["norm"] else 0),
                "flops": n * (6 + 6 * case["norm"]) if back else n * (3 + 4 * case["norm"])}
    n = T * case["V"]
    return {"bytes": n * e * (1 if case["mode"] == "loss" else 2) + T * case["top"] * (8 + e) + 12 * T, "flops": n * {"loss": 4, "step": 7, "backward": 4}[case["mode"]]}


# --------------------------------------------------------------------------- the definitions in 64 bits


def _exact_weights(s):
    """Every weight looked up byte by byte: column c of a row lies in block c / 128, in word 4 ((c % 32) / 8) + (c % 128) / 32 of
    it, in the byte and half of a byte that its place among eight neighbours says."""
    c = torch.arange(s["d_in"], device=DEVICE)
    inner = c % 8
    byte = c // 128 * 64 + (c % 32 // 8 * 4 + c % 128 // 32) * 4 + inner % 2 * 2 + inner // 4
    u = s["q"][:, byte].to(torch.int64)
    u = torch.where(inner // 2 % 2 == 1, u // 16, u % 16)
    spread = lambda v: v.double().repeat_interleave(s["group"], 1)[:, :s["d_in"]]
    zero = spread(s["zero"]) if s["zero"] is not None else 8.0
    return (u.double() - zero) * spread(s["scale"])


def _exact_turn(x, angle, s):
    """Pairs as complex numbers, times e^(i angle)."""
    half = s["rotary"] // 2
    body, rest = x[..., :2 * half], x[..., 2 * half:]
    grid = body.unflatten(-1, (half, 2)) if s["interleaved"] else body.unflatten(-1, (2, half)).transpose(-1, -2)
    turned = torch.view_as_real(torch.complex(grid[..., 0], grid[..., 1]) * torch.polar(torch.ones_like(angle), angle).unsqueeze(1))
    body = turned.flatten(-2) if s["interleaved"] else turned.transpose(-1, -2).flatten(-2)
    return torch.cat([body, rest], -1)


def _exact_rope(s):
    angle = torch.outer(s["positions"].double(), s["inv_freq"].double())
    out = {}
    for name in ("q", "k"):
        x, w = s[name].double(), s["w_" + name]
        n = torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / s["d"] + s["eps"]
        if s["op"] == "rope":
            out[name] = _exact_turn(x / n.sqrt() * w.double() if s["norm"] else x, angle, s)
            continue
        g = _exact_turn(s["d%s_out" % name].double(), -angle, s)
        if s["norm"]:
            out["dw_" + name] = torch.einsum("thd,thd->d", g, x / n.sqrt())
            g = g * w.double()
            g = g / n.sqrt() - x * torch.einsum("thd,thd->th", g, x).unsqueeze(-1) / (s["d"] * n ** 1.5)
        out["d" + name] = g
    return out


def _exact_distill(s):
    T, tau, mode = s["T"], s["tau"], s["mode"]
    loss = torch.zeros(T, dtype=torch.float64, device=DEVICE)
    lse = s["lse"].double() if mode == "backward" else torch.zeros_like(loss)
    dlogits = torch.empty(T, s["V"], dtype=torch.float64, device=DEVICE) if mode != "loss" else None
    step = max(1, (1 << 26) // s["V"])
    for i in range(0, T, step):
        rows = slice(i, min(T, i + step))
        z, ids = s["logits"][rows].double() / tau, s["ids"][rows]
        here = (ids >= 0).double()
        log_p = torch.log_softmax((s["teacher"][rows].double() / tau).masked_fill(ids < 0, -math.inf), 1)
        p = torch.exp(log_p)
        if mode != "backward":
            lse[rows] = torch.logsumexp(z, 1)
            log_q = z.gather(1, ids.clamp(min=0)) - lse[rows].reshape(-1, 1)
            loss[rows] = s["weight"][rows].double() * tau ** 2 * (p * (log_p.masked_fill(ids < 0, 0.0) - log_q) * here).sum(1)
        if mode != "loss":
            dense = torch.zeros_like(z)
            row = torch.arange(z.shape[0], device=DEVICE).reshape(-1, 1).expand_as(ids)
            dense.index_put_((row, ids.clamp(min=0)), p * here, accumulate=True)
            dlogits[rows] = (torch.exp(z - lse[rows].reshape(-1, 1)) - dense) * (s["weight"][rows].double() * tau).reshape(-1, 1)
    if mode == "backward":
        return {"dlogits": dlogits}
    return {"loss": loss, "lse": lse, "dlogits": dlogits} if mode == "step" else {"loss": loss, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "int4":
        return torch.einsum("tk,nk->tn", s["x"].double(), _exact_weights(s))
    if case["op"] == "int4_grad":
        return torch.einsum("tn,nk->tk", s["dy"].double(), _exact_weights(s))
    return _exact_distill(s) if case["op"] == "distill" else _exact_rope(s)
