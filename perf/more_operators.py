"""The rest of a student layer on packed sequences, as measured cases.

A step on a packed batch of spliced sequences looks its tokens up in the embedding, norms the rows
before each block, and lets every token attend to its own sequence: causally, with a prompt that is
seen whole, with scores capped by a tanh or lowered with the distance.  These operators, forward and
backward, stand here with their plain form (elementary torch operations in 32 bits, rounded once)
and their definition in 64 bits (exact); with `own` set, run() makes the library's calls.
"""

from __future__ import annotations

import math
import random

import torch

own = False

EPS = 1e-6  # of the rows' norms (the RMS epsilon of the synthetic hidden rows)

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    att = lambda name, op, T, hq, hk, D, **kw: dict(
        dict(name=name, op=op, T=T, hq=hq, hk=hk, D=D, seqs=1, pad=0, causal=True, prefix=0.0, cap=0.0, bias=False), **kw)
    norm = lambda name, op, T, d, **kw: dict(
        dict(name=name, op=op, T=T, d=d, kind="layer", bias=True, residual=False, dtype="bf16"), **kw)
    emb = lambda name, op, T, V, d, **kw: dict(dict(name=name, op=op, T=T, V=V, d=d, dtype="bf16"), **kw)
    return [
        # one short sequence of a tiny student: launches and host time
        att("att_tiny", "att", 100, 4, 2, 64),
        # scoring one rollout: a prompt, a 4096-token prefix and a 1024-token continuation
        att("att_score", "att", 5633, 32, 8, 128),
        # one long trace with a bias that falls with the distance
        att("att_long_bias", "att", 20011, 8, 2, 128, bias=True),
        # training on 8 x 4096 packed tokens
        att("att_step_batch", "att_step", 32768, 32, 8, 128, seqs=8),
        # a ragged micro-batch whose prompts are seen whole, capped scores, rows behind the last sequence
        att("att_step_prefix_cap", "att_step", 5003, 15, 3, 96, seqs=7, pad=117, prefix=0.5, cap=30.0),
        # many turns of some forty tokens each, every token sees its whole turn
        att("att_step_turns", "att_step", 8192, 16, 16, 64, seqs=200, causal=False),
        # one token of each of 64 prompts
        norm("norm_tokens_64", "norm", 64, 4096),
        # training on 8 x 4096 packed tokens, the residual added on the way
        norm("norm_step_batch", "norm_step", 32768, 4096, residual=True),
        # fp32 rows of a width that no power of two divides, without centring
        norm("norm_step_rms_f32", "norm_step", 3001, 2040, kind="rms", bias=False, dtype="f32"),
        # one token of each of 64 prompts
        emb("emb_tokens_64", "emb", 64, 151936, 4096),
        # training on 8 x 4096 packed tokens of a full vocabulary
        emb("emb_step_batch", "emb_step", 32768, 151936, 4096),
        # fp32 rows of a small vocabulary: every id many times
        emb("emb_step_small_f32", "emb_step", 9001, 4097, 1000, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


#: token pairs times query heads that the largest listed case's plain form holds
MOST_PAIRS = 8 * 4096 * 4096 * 32


def draw(rng):
    op = rng.choice(("att", "att", "att_step", "att_step", "att_step", "norm", "norm_step", "norm_step",
                     "emb", "emb_step", "emb_step"))
    if op.startswith("att"):
        hk = rng.choice((1, 2, 3, 4, 8))
        hq = hk * rng.choice((1, 1, 2, 4, 5))
        T = _log_int(rng, 1, 16384)
        c = dict(op=op, T=T, hq=hq, hk=hk, D=rng.choice((32, 64, 80, 96, 128, 128)), seqs=min(T, _log_int(rng, 1, 64)),
                 pad=rng.choice((0, 0, 1, 60)), causal=rng.random() < 0.8, prefix=rng.choice((0.0, 0.0, 0.4)),
                 cap=rng.choice((0.0, 0.0, 30.0)), bias=rng.random() < 0.3)
        while _pairs_held(c) * hq > MOST_PAIRS:
            c["T"] = c["T"] * 3 // 4
        c["seqs"] = min(c["T"], c["seqs"])
        return c
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op.startswith("norm"):
        d = 8 * _log_int(rng, 8, 1024)
        T = _log_int(rng, 1, 32768)
        while T * d > 32768 * 2048:
            T //= 2
        return dict(op=op, T=T, d=d, kind=rng.choice(("layer", "layer", "rms")), bias=rng.random() < 0.6,
                    residual=rng.random() < 0.4, dtype=dtype)
    d, T = 8 * _log_int(rng, 8, 512), _log_int(rng, 1, 32768)
    V = _log_int(rng, 64, 151936)
    while (T + V) * d > 100000 * 4096:
        T, V = max(1, T // 2), V // 2
    return dict(op=op, T=T, V=V, d=d, dtype=dtype)


# ---------------------------------------------------------------- inputs ---

def _lengths(c):
    """Lengths of the packed sequences of a case, the same for every seed: equal ones where they
    divide the batch, else drawn ones."""
    T, n = c["T"], c["seqs"]
    if n > 1 and T % n == 0 and T // n >= 1024:
        return [T // n] * n
    rng = random.Random("%d %d" % (T, n))
    cuts = sorted(rng.sample(range(1, T), n - 1)) if n > 1 else []
    return [b - a for a, b in zip([0] + cuts, cuts + [T])]


def _prefixes(c):
    """Tokens at each sequence's beginning that all its tokens see."""
    return [int(n * c["prefix"]) for n in _lengths(c)]


def _pairs_held(c):
    """Token pairs a head has in the plain form: sequences padded to the longest, or all tokens at once."""
    lens = _lengths(c)
    return min(len(lens) * max(lens) ** 2, c["T"] ** 2)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    s = dict(c=c)
    if c["op"].startswith("att"):
        T, hq, hk, D = c["T"] + c["pad"], c["hq"], c["hk"], c["D"]
        bf = lambda t: t.to(torch.bfloat16)
        # heads after their norm (unit rows times weights: some heads sharper), values as projected
        qk = randn(T, hq + hk, D) * (0.8 + 0.8 * torch.rand(hq + hk, 1, generator=gen, device="cuda"))
        s["q"], s["k"] = bf(qk[:, :hq]), bf(qk[:, hq:])
        qkv = bf(randn(T, hq + 2 * hk, D))  # values are a view of the fused projection
        s["v"] = qkv[:, hq + hk:]
        lens = _lengths(c)
        cu = [0]
        for n in lens:
            cu.append(cu[-1] + n)
        s["cu"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
        s["prefix_end"] = None
        if c["prefix"]:
            ends = [a + p for a, p in zip(cu, _prefixes(c))]
            s["prefix_end"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
        s["slopes"] = None
        if c["bias"]:  # a geometric sequence, as distance biases have
            s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, hq + 1, device="cuda", dtype=torch.float32) / hq)
        if c["op"] == "att_step":
            s["do"] = bf(randn(T, hq, D) * 0.01)
        return s
    dt = DTYPES[c["dtype"]]
    T, d = c["T"], c["d"]
    if c["op"].startswith("norm"):
        # rows of the residual stream: of different sizes, with an offset
        x = randn(T, d) * (0.5 + 3 * torch.rand(T, 1, generator=gen, device="cuda")) + 0.3 * randn(T, 1)
        s["x"] = x.to(dt)
        s["residual"] = randn(T, d).to(dt) if c["residual"] else None
        s["w"] = (1 + 0.2 * randn(d)).to(dt)
        s["b"] = (0.2 * randn(d)).to(dt) if c["bias"] else None
        if c["op"] == "norm_step":
            s["dy"] = (randn(T, d) * 0.01).to(dt)
            s["dh"] = (randn(T, d) * 0.01).to(dt) if c["residual"] else None
        return s
    V = c["V"]
    s["W"] = (randn(V, d) * 0.02).to(dt)
    # ids by falling frequency, as a text's: the k-th with a probability of about 1 / (k ln V)
    u = torch.rand(T, generator=gen, device="cuda", dtype=torch.float64)
    s["ids"] = (torch.exp(u * math.log(V + 1)) - 1).long().clamp(0, V - 1).to(torch.int32)
    s["scale"] = d ** 0.5
    if c["op"] == "emb_step":
        s["dy"] = (randn(T, d) * 0.01).to(dt)
    return s


# ------------------------------------------------------------ plain forms ---

def _batched(s):
    """Token index, position and sequence of a [batch, length] layout of the packed tokens, -1 where
    there is none: a sequence a batch entry, or all tokens in one where that holds fewer pairs."""
    c = s["c"]
    cu = s["cu"].long()
    T, S = c["T"], c["seqs"]
    t = torch.arange(T, device="cuda")
    seq = torch.bucketize(t, cu[1:], right=True)
    if S * max(_lengths(c)) ** 2 > T * T:
        return t[None], (t - cu[seq])[None], seq[None]
    pos = torch.arange(max(_lengths(c)), device="cuda")
    at = cu[:-1, None] + pos
    there = at < cu[1:, None]
    seq = torch.arange(S, device="cuda")[:, None].expand_as(at)
    return torch.where(there, at, -1), pos.expand_as(at), torch.where(there, seq, -1)


def _plain_att(s, step):
    c = s["c"]
    q, k, v = s["q"], s["k"], s["v"]
    rows, hq, D = q.shape
    hk = k.shape[1]
    scale = 1 / math.sqrt(D)
    index, pos, seq = _batched(s)
    there = index >= 0
    b, n = index.shape
    # [batch, key heads, queries of a key head, tokens, D]
    take = lambda x: x.float()[index.clamp(min=0)].permute(0, 2, 1, 3).reshape(b, hk, -1, n, D) * there[:, None, None, :, None]
    Q, K, Vv = take(q), take(k), take(v)
    seen = (seq[:, :, None] == seq[:, None]) & there[:, :, None] & there[:, None]
    if c["causal"]:
        ahead = pos[:, None] > pos[:, :, None]
        if s["prefix_end"] is not None:
            length = (s["prefix_end"] - s["cu"][:-1]).long()[seq.clamp(min=0)]
            ahead &= pos[:, None] >= length[:, None]
        seen &= ~ahead
    seen = seen[:, None, None]
    z = (Q * scale) @ K.transpose(-1, -2)
    bend = None
    if c["cap"]:
        bend = (z / c["cap"]).tanh()
        z = bend * c["cap"]
    if s["slopes"] is not None:
        far = (pos[:, :, None] - pos[:, None]).abs().float()[:, None, None]
        z = z - s["slopes"].reshape(1, hk, -1, 1, 1) * far
    z = z.masked_fill(~seen, -math.inf)
    top = z.amax(-1, keepdim=True).clamp(min=-1e30)
    p = (z - top).exp()
    total = p.sum(-1, keepdim=True)
    lse = top + total.log()
    p = p / total.clamp(min=1e-30)
    o = p @ Vv

    def back(x):  # into the packed layout, 0 behind the last sequence
        out = torch.zeros((rows, x.shape[1] * x.shape[2], D), device="cuda")
        out[index[there]] = x.permute(0, 3, 1, 2, 4).reshape(b, n, -1, D)[there]
        return out.to(q.dtype)

    got = dict(o=back(o), lse=torch.full((hq, rows), -math.inf, device="cuda"))
    got["lse"][:, index[there]] = lse[..., 0].permute(0, 3, 1, 2).reshape(b, n, hq)[there].t()
    if not step:
        return got
    do = take(s["do"])
    dp = do @ Vv.transpose(-1, -2)
    got["dv"] = back((p.transpose(-1, -2) @ do).sum(2, keepdim=True))
    dz = p * (dp - (p * dp).sum(-1, keepdim=True))
    if bend is not None:
        dz = dz * (1 - bend * bend)
    got["dq"] = back(dz @ K * scale)
    got["dk"] = back((dz.transpose(-1, -2) @ Q).sum(2, keepdim=True) * scale)
    return got


def _plain_norm(s, step):
    c = s["c"]
    dt, w = s["x"].dtype, s["w"].float()
    h = s["x"]
    if s["residual"] is not None:
        h = (h.float() + s["residual"].float()).to(dt)
    f = h.float()
    if c["kind"] == "layer":
        f = f - f.mean(-1, keepdim=True)
    inv = (f.square().mean(-1, keepdim=True) + EPS).rsqrt()
    n = f * inv
    y = n * w
    if s["b"] is not None:
        y = y + s["b"].float()
    got = dict(y=y.to(dt))
    if s["residual"] is not None:
        got["h"] = h
    if not step:
        return got
    dy = s["dy"].float()
    a = dy * w
    dx = a - n * (a * n).mean(-1, keepdim=True)
    if c["kind"] == "layer":
        dx = dx - a.mean(-1, keepdim=True)
    dx = dx * inv
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    got.update(dx=dx.to(dt), dw=(dy * n).sum(0))
    if s["b"] is not None:
        got["db"] = dy.sum(0)
    return got


def _plain_emb(s, step):
    W, ids = s["W"], s["ids"].long()
    y = (W[ids].float() * s["scale"]).to(W.dtype)
    if not step:
        return y
    dW = torch.zeros(W.shape, device="cuda").index_add_(0, ids, s["dy"].float())
    return dict(y=y, dW=(dW * s["scale"]).to(W.dtype))


# ------------------------------------------------------------ the library ---

def _own_att(s, step):
    from paper_2609_36246_gb300 import binding as B

    more = dict(causal=s["c"]["causal"], prefix_end=s["prefix_end"], cap=s["c"]["cap"], slopes=s["slopes"])
    o, lse = B.olive_packed_attention_fwd(s["q"], s["k"], s["v"], s["cu"], **more)
    if not step:
        return dict(o=o, lse=lse)
    dq, dk, dv = B.olive_packed_attention_bwd(s["do"], s["q"], s["k"], s["v"], o, lse, s["cu"], **more)
    return dict(o=o, lse=lse, dv=dv, dq=dq, dk=dk)


def _own_norm(s, step):
    from paper_2609_36246_gb300 import binding as B

    kind = s["c"]["kind"]
    y, h, stats = B.olive_row_norm_fwd(s["x"], s["w"], s["b"], residual=s["residual"], eps=EPS, kind=kind, save=step)
    got = dict(y=y)
    if s["residual"] is not None:
        got["h"] = h
    if not step:
        return got
    got["dx"], got["dw"], db = B.olive_row_norm_bwd(s["dy"], h, s["w"], stats, g_h=s["dh"], kind=kind,
                                                    need_db=s["b"] is not None)
    if s["b"] is not None:
        got["db"] = db
    return got


def _own_emb(s, step):
    from paper_2609_36246_gb300 import binding as B

    y = B.olive_embedding_fwd(s["W"], s["ids"], scale=s["scale"])
    if not step:
        return y
    dW = B.olive_embedding_bwd(s["dy"], s["ids"], s["c"]["V"], scale=s["scale"], grad_dtype=s["W"].dtype)
    return dict(y=y, dW=dW)


def run(state):
    op = state["c"]["op"]
    step = op.endswith("_step")
    if op.startswith("att"):
        return _own_att(state, step) if own else _plain_att(state, step)
    if op.startswith("norm"):
        return _own_norm(state, step) if own else _plain_norm(state, step)
    return _own_emb(state, step) if own else _plain_emb(state, step)


def _pairs_seen(c):
    """Pairs of tokens that a head's scores are made of."""
    if not c["causal"]:
        return sum(n * n for n in _lengths(c))
    # a prefix's tokens see all of it, the others what is not ahead
    return sum(p * p + (n * (n + 1) - p * (p + 1)) // 2 for n, p in zip(_lengths(c), _prefixes(c)))


def work(case):
    """Inputs read once, outputs written once, products computed once (scores again in a backward)."""
    c = case
    step = c["op"].endswith("_step")
    if c["op"].startswith("att"):
        T, hq, hk, D = c["T"] + c["pad"], c["hq"], c["hk"], c["D"]
        q, kv = 2.0 * T * hq * D, 2.0 * T * hk * D
        size = 2 * q + 2 * kv + 4.0 * hq * T
        flops = 4.0 * D * hq * _pairs_seen(c)
        return dict(bytes=size + (2 * q + 2 * kv if step else 0), flops=3.5 * flops if step else flops)
    T, d = c["T"], c["d"]
    e = 4 if c["dtype"] == "f32" else 2
    row = float(e) * T * d
    if c["op"].startswith("norm"):
        both = 2 if c["residual"] else 1
        # a row's mean, its square's mean and the result: about 8 operations an element, twice that back
        return dict(bytes=row * (2 * both + (1 + both if step else 0)) + 2 * e * d,
                    flops=(24.0 if step else 8.0) * T * d)
    V = c["V"]
    # rows that T such ids are expected to name
    k = torch.arange(1, V + 1, dtype=torch.float64)
    share = torch.log1p(1 / k) / math.log(V + 1)
    named = float((1 - (1 - share) ** T).sum())
    size = 4.0 * T + e * named * d + row
    return dict(bytes=size + (row + float(e) * V * d if step else 0), flops=(2.0 if step else 1.0) * T * d)


# ------------------------------------------------- definitions in 64 bits ---

def _exact_att(s, step):
    c = s["c"]
    q, k, v = s["q"], s["k"], s["v"]
    rows, hq, D = q.shape
    hk = k.shape[1]
    per = hq // hk
    zero = lambda x: torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    got = dict(o=zero(q), lse=torch.full((hq, rows), -math.inf, dtype=torch.float64, device="cuda"))
    if step:
        got.update(dv=zero(v), dq=zero(q), dk=zero(k))
    start = 0
    for n, p in zip(_lengths(c), _prefixes(c)):
        span = slice(start, start + n)
        start += n
        at = torch.arange(n, device="cuda")
        hidden = torch.zeros(n, n, dtype=torch.bool, device="cuda")
        if c["causal"]:
            hidden = (at[None] > at[:, None]) & (at[None] >= p)
        for g in range(hk):
            mine = slice(g * per, (g + 1) * per)
            leaf = [x.double().transpose(0, 1).contiguous().requires_grad_(step) for x in (q[span, mine], k[span, g:g + 1], v[span, g:g + 1])]
            z = torch.einsum("hid,gjd->hij", leaf[0], leaf[1]) / math.sqrt(D)
            if c["cap"]:
                z = c["cap"] * torch.tanh(z / c["cap"])
            if s["slopes"] is not None:
                z = z - s["slopes"][mine].double()[:, None, None] * (at[:, None] - at[None]).abs()
            z = z.masked_fill(hidden, -math.inf)
            y = torch.einsum("hij,gjd->hid", z.softmax(-1), leaf[2])
            got["o"][span, mine] = y.detach().transpose(0, 1)
            got["lse"][mine, span] = torch.logsumexp(z.detach(), -1)
            if step:
                grads = torch.autograd.grad(y, leaf, s["do"][span, mine].double().transpose(0, 1))
                got["dq"][span, mine] = grads[0].transpose(0, 1)
                got["dk"][span, g] = grads[1][0]
                got["dv"][span, g] = grads[2][0]
            del z, y
    return got


def _exact_norm(s, step):
    c = s["c"]
    d = c["d"]
    h = s["x"].double()
    got = {}
    if s["residual"] is not None:
        full = h + s["residual"].double()
        h = full.to(s["x"].dtype).double()  # the norm is that of the sum as it is kept
    h = h.requires_grad_(step)
    w = s["w"].double().requires_grad_(step)
    b = None if s["b"] is None else s["b"].double().requires_grad_(step)
    if c["kind"] == "layer":
        y = torch.nn.functional.layer_norm(h, (d,), w, b, EPS)
    else:
        y = w * h / (h.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
        y = y if b is None else y + b
    got["y"] = y.detach()
    if s["residual"] is not None:
        got["h"] = full
    if step:
        leaf = [h, w] + ([] if b is None else [b])
        grads = torch.autograd.grad(y, leaf, s["dy"].double())
        got["dx"] = grads[0] + (0 if s["dh"] is None else s["dh"].double())
        got["dw"] = grads[1]
        if b is not None:
            got["db"] = grads[2]
    return got


def _exact_emb(s, step):
    ids = s["ids"].long()
    y = torch.nn.functional.embedding(ids, s["W"]).double() * s["scale"]
    if not step:
        return y
    # tokens in the order of their ids, summed up to each row's end
    order = ids.argsort(stable=True)
    named, count = torch.unique_consecutive(ids[order], return_counts=True)
    dW = torch.zeros(s["W"].shape, dtype=torch.float64, device="cuda")
    dW[named] = torch.segment_reduce(s["dy"].double()[order], "sum", lengths=count, axis=0) * s["scale"]
    return dict(y=y, dW=dW)


def exact(case, seed):
    s = prepare(dict(case), seed)
    step = case["op"].endswith("_step")
    if case["op"].startswith("att"):
        return _exact_att(s, step)
    return _exact_norm(s, step) if case["op"].startswith("norm") else _exact_emb(s, step)
