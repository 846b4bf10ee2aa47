"""What a student's trainer runs around the LM-head loss, as measured cases.

The library's hidden rows come out of a decoder layer and its gradients go into an optimiser.  The
operators here are the parts of that way that a packed batch of spliced sequences needs beside the
loss: the norm of each head's queries and keys with the rotation by the token's position in its
sequence, the gated feed-forward block, and the clipping of all gradients by their global norm.

Every operator has its plain form here (elementary torch operations in 32 bits, rounded once) and
its definition in 64 bits (exact); with `own` set, run() makes the library's calls.
"""

from __future__ import annotations

import math
import random

import torch

own = False

EPS = 1e-6        # of the heads' norms (the RMS epsilon of the synthetic hidden rows)
W_STD = 0.02      # standard deviation of weight matrices (synth.py)
BASE = 1000000.0  # rotary base of long-context students

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    mlp = lambda name, op, T, d, f, **kw: dict(
        dict(name=name, op=op, T=T, d=d, f=f, act="silu", residual=True), **kw)
    qk = lambda name, op, T, hq, hk, D, **kw: dict(
        dict(name=name, op=op, T=T, hq=hq, hk=hk, D=D, R=D, interleaved=False, seqs=1, dtype="bf16"), **kw)
    clip = lambda name, **kw: dict(
        dict(name=name, op="clip", layers=1, d=256, f=704, V=0, dtype="bf16", limit=1.0, scale=1.0), **kw)
    return [
        # one token of one rollout through a d = 4096 block: the weights are read once
        mlp("mlp_token", "mlp", 1, 4096, 12288),
        # one token of each of 64 prompts, d = 2048
        mlp("mlp_tokens_64", "mlp", 64, 2048, 6144),
        # scoring one rollout's odd-sized continuation, the tanh form of GELU, no residual
        mlp("mlp_continuation", "mlp", 1003, 2560, 6912, act="gelu_tanh", residual=False),
        # the smallest training step (4 x 128 tokens, d = 256): launches and host time
        mlp("mlp_step_tiny", "mlp_step", 512, 256, 704),
        # training on one ragged micro-batch, widths that no tile divides
        mlp("mlp_step_ragged", "mlp_step", 2777, 2040, 5464),
        # training on 2 x 4096 packed tokens at d = 4096
        mlp("mlp_step_batch", "mlp_step", 8192, 4096, 12288),
        # one token: 32 query and 8 key heads of 128
        qk("qk_token", "qk", 1, 32, 8, 128),
        # training on 8 x 4096 packed tokens, forward and backward
        qk("qk_step_batch", "qk_step", 32768, 32, 8, 128, seqs=8),
        # part of an odd head rotated, neighbours paired, fp32, one key head
        qk("qk_step_partial", "qk_step", 3001, 12, 1, 80, R=32, interleaved=True, seqs=3, dtype="f32"),
        # gradients of one tiny layer: launches and host time
        clip("clip_tiny", scale=30.0),
        # gradients of two layers and of a full vocabulary's LM head at d = 4096
        clip("clip_batch", layers=2, d=4096, f=12288, V=151936, scale=3.0),
        # fp32 gradients of four layers, odd widths, below the limit
        clip("clip_f32_below", layers=4, d=1001, f=2735, V=4096, dtype="f32", limit=1e6),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _not_3072(n, step):
    return n + step if n == 3072 else n


def draw(rng):
    op = rng.choice(("mlp", "mlp", "mlp_step", "mlp_step", "qk", "qk_step", "qk_step", "clip", "clip"))
    if op.startswith("mlp"):
        return dict(op=op, T=_not_3072(_log_int(rng, 1, 8192), 1), d=_not_3072(8 * _log_int(rng, 32, 512), 8),
                    f=_not_3072(8 * _log_int(rng, 64, 1536), 8), act=rng.choice(("silu", "silu", "gelu_tanh")),
                    residual=rng.random() < 0.6)
    if op.startswith("qk"):
        D = rng.choice((64, 80, 96, 128, 128, 256))
        hk = rng.choice((1, 2, 4, 5, 8))
        T = _not_3072(_log_int(rng, 1, 32768), 1)
        hq = hk * rng.choice((1, 2, 4, 5))
        while T * (hq + hk) * D > 32768 * 40 * 128:
            T //= 2
        return dict(op=op, T=T, hq=hq, hk=hk, D=D, R=rng.choice((D, D, D, D // 2, 32)),
                    interleaved=rng.random() < 0.3, seqs=min(T, _log_int(rng, 1, 64)),
                    dtype=rng.choice(("bf16", "bf16", "bf16", "f32")))
    d = _not_3072(_log_int(rng, 64, 4096), 1)
    return dict(op=op, layers=rng.randint(1, 5), d=d, f=_not_3072(_log_int(rng, 2 * d, 3 * d), 1),
                V=rng.choice((0, _log_int(rng, 512, 100003))), dtype=rng.choice(("bf16", "bf16", "f32", "mixed")),
                limit=rng.choice((1.0, 0.5, 1e6)), scale=math.exp(rng.uniform(-3.0, 5.0)))


# ---------------------------------------------------------------- inputs ---

def _lengths(c):
    """Lengths of the packed sequences of a case, the same for every seed."""
    rng = random.Random("%d %d" % (c["T"], c["seqs"]))
    cuts = sorted(rng.sample(range(1, c["T"]), c["seqs"] - 1)) if c["seqs"] > 1 else []
    return [b - a for a, b in zip([0] + cuts, cuts + [c["T"]])]


def _shapes(c):
    """Shapes and dtypes of a case's gradients: a layer's matrices, its norms' weights (fp32, as
    the library gives them), then the LM head."""
    d, f = c["d"], c["f"]
    whole = [(d + 2 * max(8, d // 4), d), (d, d), (f, d), (f, d), (d, f)]
    small = [(d,), (d,), (128,), (128,)]
    main = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    head = torch.float32 if c["dtype"] == "mixed" else main
    got = [(s, main) for _ in range(c["layers"]) for s in whole]
    got += [(s, torch.float32) for _ in range(c["layers"]) for s in small]
    return got + ([((c["V"], d), head)] if c["V"] else [])


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    s = dict(c=c)
    if c["op"].startswith("mlp"):
        T, d, f = c["T"], c["d"], c["f"]
        bf = lambda t: t.to(torch.bfloat16)
        x = randn(T, d)
        s["x"] = bf(x * (x.square().mean(1, keepdim=True) + EPS).rsqrt())
        # student weights: pre-activations of a spread of about one
        s["W_gate"], s["W_up"] = bf(randn(f, d) * (1.3 / math.sqrt(d))), bf(randn(f, d) * (1.3 / math.sqrt(d)))
        s["W_down"] = bf(randn(d, f) * W_STD)
        s["residual"] = bf(randn(T, d)) if c["residual"] else None
        if c["op"] == "mlp_step":
            s["dy"] = bf(randn(T, d) * (0.1 / math.sqrt(T)))
        return s
    if c["op"].startswith("qk"):
        T, hq, hk, D, R, dt = c["T"], c["hq"], c["hk"], c["D"], c["R"], DTYPES[c["dtype"]]
        # one fused projection: queries, keys and values of a token side by side, some heads larger
        qkv = randn(T, hq + 2 * hk, D) * (0.3 + 3 * torch.rand(hq + 2 * hk, 1, generator=gen, device="cuda"))
        s["qkv"] = qkv.to(dt)
        s["q"], s["k"] = s["qkv"][:, :hq], s["qkv"][:, hq:hq + hk]
        s["w_q"], s["w_k"] = (1 + 0.2 * randn(D)).to(dt), (1 + 0.2 * randn(D)).to(dt)
        lens = _lengths(c)
        start = torch.randint(0, 4096, (1,), generator=gen, device="cuda") if T == 1 else 0
        pos = torch.cat([torch.arange(n, device="cuda") for n in lens]) + start
        s["positions"] = pos.to(torch.int32)
        rows = max(lens) if T > 1 else 4096
        angle = torch.arange(rows, device="cuda").double()[:, None] * BASE ** (
            -torch.arange(0, R, 2, device="cuda").double() / R)
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        if c["op"] == "qk_step":
            s["dq"], s["dk"] = (randn(T, hq, D) * 0.01).to(dt), (randn(T, hk, D) * 0.01).to(dt)
        return s
    shapes = _shapes(c)
    total = sum(math.prod(x) for x, _ in shapes)
    spread = c["scale"] / math.sqrt(total)
    s["grads"] = [(randn(*x) * spread).to(t) for x, t in shapes]
    s["out"] = [torch.empty_like(g) for g in s["grads"]]
    return s


# ------------------------------------------------------------ plain forms ---

def _activation(g, act):
    """The activation and its derivative."""
    if act == "silu":
        e = 1 / (1 + (-g).exp())
        return g * e, e * (1 + g * (1 - e))
    k = math.sqrt(2 / math.pi)
    t = (k * (g + 0.044715 * g * g * g)).tanh()
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)


def _plain_mlp(s, step):
    x, wg, wu, wd = (s[k].float() for k in ("x", "W_gate", "W_up", "W_down"))
    g, u = x @ wg.t(), x @ wu.t()
    a, slope = _activation(g, s["c"]["act"])
    h = a * u
    y = h @ wd.t()
    if s["residual"] is not None:
        y = y + s["residual"].float()
    r = lambda t: t.to(torch.bfloat16)
    if not step:
        return r(y)
    dy = s["dy"].float()
    dh = dy @ wd
    dg, du = dh * u * slope, dh * a
    return dict(y=r(y), dx=r(dg @ wg + du @ wu), dW_gate=r(dg.t() @ x), dW_up=r(du.t() @ x), dW_down=r(dy.t() @ h))


def _pairs(x, R, interleaved):
    """The two members of each rotated pair."""
    return (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., :R // 2], x[..., R // 2:R])


def _joined(a, b, rest, interleaved):
    both = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((both, rest), -1)


def _plain_qk(s, step):
    c = s["c"]
    R, inter = c["R"], c["interleaved"]
    cos, sin = (s[k][s["positions"].long()][:, None] for k in ("cos", "sin"))
    out = {}
    for name, x, w in (("q", s["q"], s["w_q"]), ("k", s["k"], s["w_k"])):
        dt, x, w = x.dtype, x.float(), w.float()
        inv = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
        n = x * inv
        a, b = _pairs(n * w, R, inter)
        out[name] = _joined(a * cos - b * sin, b * cos + a * sin, (n * w)[..., R:], inter).to(dt)
        if step:
            dy = s["d" + name].float()
            a, b = _pairs(dy, R, inter)
            dn = _joined(a * cos + b * sin, b * cos - a * sin, dy[..., R:], inter)
            out["dw_" + name] = (dn * n).sum((0, 1))
            dn = dn * w
            out["d" + name] = (inv * (dn - n * (dn * n).mean(-1, keepdim=True))).to(dt)
    return out


def _plain_clip(s):
    grads, limit = s["grads"], s["c"]["limit"]
    norm = torch.stack([g.float().square().sum() for g in grads]).sum().sqrt()
    factor = (limit / (norm + 1e-6)).clamp(max=1.0)
    return dict(norm=norm.reshape(1), grads=[(g.float() * factor).to(g.dtype) for g in grads])


# ------------------------------------------------------------ the library ---

def _own_mlp(s, step):
    from paper_2609_36246_gb300 import binding as B

    w, act = (s["W_gate"], s["W_up"], s["W_down"]), s["c"]["act"]
    y, saved = B.olive_gated_mlp_fwd(s["x"], *w, residual=s["residual"], act=act, save=step)
    if not step:
        return y
    dx, dg, du, dd = B.olive_gated_mlp_bwd(s["dy"], s["x"], *w, saved, act=act)
    return dict(y=y, dx=dx, dW_gate=dg, dW_up=du, dW_down=dd)


def _own_qk(s, step):
    from paper_2609_36246_gb300 import binding as B

    more = (s["w_q"], s["w_k"], s["cos"], s["sin"], s["positions"], EPS, s["c"]["interleaved"])
    q, k = B.olive_qk_norm_rope_fwd(s["q"], s["k"], *more)
    if not step:
        return dict(q=q, k=k)
    dq, dk, dw_q, dw_k = B.olive_qk_norm_rope_bwd(s["dq"], s["dk"], s["q"], s["k"], *more)
    return dict(q=q, k=k, dq=dq, dk=dk, dw_q=dw_q, dw_k=dw_k)


def _own_clip(s):
    from paper_2609_36246_gb300 import binding as B

    norm = B.olive_grad_clip(s["grads"], s["c"]["limit"], out=s["out"])
    return dict(norm=norm, grads=s["out"])


def run(state):
    op = state["c"]["op"]
    if op == "clip":
        return _own_clip(state) if own else _plain_clip(state)
    step = op.endswith("_step")
    if op.startswith("mlp"):
        return _own_mlp(state, step) if own else _plain_mlp(state, step)
    return _own_qk(state, step) if own else _plain_qk(state, step)


def work(case):
    """Inputs read once, outputs written once, products computed once."""
    c = case
    if c["op"].startswith("mlp"):
        T, d, f = c["T"], c["d"], c["f"]
        rows, weights = 2.0 * T * d, 6.0 * d * f
        if c["op"] == "mlp":
            return dict(bytes=(2 + c["residual"]) * rows + weights, flops=6.0 * T * d * f)
        return dict(bytes=(4 + c["residual"]) * rows + 2 * weights, flops=18.0 * T * d * f)
    if c["op"].startswith("qk"):
        e = 4 if c["dtype"] == "f32" else 2
        n = e * c["T"] * (c["hq"] + c["hk"]) * c["D"]
        tables = 4 * c["T"] + 4 * c["R"] * (max(_lengths(c)) if c["T"] > 1 else 1)
        step = c["op"] == "qk_step"
        # a pair's rotation and its norm: about 10 operations an element each way
        return dict(bytes=float((4 if step else 2) * n + tables), flops=(30.0 if step else 10.0) * n / e)
    size = sum(math.prod(x) * t.itemsize for x, t in _shapes(c))
    return dict(bytes=2.0 * size, flops=3.0 * sum(math.prod(x) for x, _ in _shapes(c)))


# ------------------------------------------------- definitions in 64 bits ---

def _exact_mlp(s, step):
    names = ("x", "W_gate", "W_up", "W_down")
    x, wg, wu, wd = leaf = [s[k].double().requires_grad_(step) for k in names]
    F = torch.nn.functional
    act = F.silu if s["c"]["act"] == "silu" else lambda t: F.gelu(t, approximate="tanh")
    y = F.linear(act(F.linear(x, wg)) * F.linear(x, wu), wd)
    if s["residual"] is not None:
        y = y + s["residual"].double()
    if not step:
        return y
    got = torch.autograd.grad(y, leaf, s["dy"].double())
    return dict(y=y.detach(), **dict(zip(("dx", "dW_gate", "dW_up", "dW_down"), got)))


def _exact_qk(s, step):
    c = s["c"]
    R, half = c["R"], c["R"] // 2
    p = s["positions"].long()
    turn = torch.complex(s["cos"].double(), s["sin"].double())[p][:, None]  # e^(i angle) of each pair
    order = torch.arange(R, device="cuda").reshape((half, 2) if c["interleaved"] else (2, half))
    order = order if c["interleaved"] else order.t()  # [pair, member]
    out = {}
    for name in ("q", "k"):
        x, w = (s[k].double().requires_grad_(step) for k in (name, "w_" + name))
        n = w * x / (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
        z = torch.view_as_real(torch.view_as_complex(n[..., order].contiguous()) * turn)
        y = n.clone()
        y[..., order.reshape(-1)] = z.flatten(-2)
        out[name] = y.detach()
        if step:
            out["d" + name], out["dw_" + name] = torch.autograd.grad(y, (x, w), s["d" + name].double())
    return out


def exact(case, seed):
    s = prepare(dict(case), seed)
    op = case["op"]
    if op == "clip":
        parts = [torch.linalg.vector_norm(g.double()) for g in s["grads"]]
        norm = torch.linalg.vector_norm(torch.stack(parts)).reshape(1)
        factor = min(1.0, case["limit"] / (float(norm) + 1e-6))
        return dict(norm=norm, grads=[g.double() * factor for g in s["grads"]])
    step = op.endswith("_step")
    return _exact_mlp(s, step) if op.startswith("mlp") else _exact_qk(s, step)
