"""Attention inside packed sequences against the definition in 64 bits.

Tolerances.  A score is a sum of up to 128 exact products in fp32: off by at most 2^-16 of A, the
largest sum of the magnitudes of a row's products (times the scale), whatever the order; the bias and
the cap add 2^-22 of their size each, and an exponential is off by its argument's error.  The weights
are rounded to bf16, 2^-8 of each, so an output is within (2^-8 + 2^-15 (A + B)) of the sum of its
terms' magnitudes, and its own rounding, 2^-8 of it.
"""

import math

import pytest
import torch

from paper_2609_36246_gb300 import binding as B

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
STEP = 2.0 ** -8 * 1.01
# A weight (of a row whose largest is near 1) or a product below the smallest normal number may count as 0.
FLUSH = 2.0 ** -126


def _case(lens, hq, hk, D, pad=0, prefix=None, cap=0.0, bias=False, causal=True, seed=0, sharp=1.0, scale=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    T = sum(lens) + pad
    qkv = (r(T, hq + 2 * hk, D) * sharp).to(BF16)
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    s = dict(q=qkv[:, :hq], k=qkv[:, hq:hq + hk], v=qkv[:, hq + hk:], do=r(T, hq, D).to(BF16), lens=lens,
             cu=torch.tensor(cu, dtype=torch.int32, device="cuda"),
             more=dict(causal=causal, cap=cap, scale=scale, prefix_end=None, slopes=None))
    if prefix is not None:
        ends = [a + min(n, prefix) for a, n in zip(cu, lens)]
        s["more"]["prefix_end"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
    if bias:
        s["more"]["slopes"] = 0.3 * 2.0 ** -torch.arange(hq, device="cuda", dtype=torch.float32)
    return s


def _seen(s, T):
    """Which key each row sees [T, T], and the rows' distances."""
    cu = s["cu"].long()
    t = torch.arange(T, device="cuda")
    seq = torch.bucketize(t, cu[1:], right=True)
    live = t < cu[-1]
    seen = (seq[:, None] == seq[None]) & live[:, None] & live[None]
    if s["more"]["causal"]:
        ok = t[None] <= t[:, None]
        end = s["more"]["prefix_end"]
        if end is not None:
            ok = ok | (t[None] < end.long()[seq.clamp(max=end.numel() - 1)][:, None])
        seen = seen & ok
    return seen, (t[:, None] - t[None]).abs().double()


def _reference(s, grads=False):
    """o and lse, gradients, and what bounds the errors, head by head."""
    q, k, v = s["q"], s["k"], s["v"]
    T, hq, D = q.shape
    per = hq // k.shape[1]
    m = s["more"]
    scale = m["scale"] or D ** -0.5
    seen, far = _seen(s, T)
    out = {n: torch.zeros(x.shape, dtype=torch.float64, device="cuda") for n, x in
           (("o", q), ("tol_o", q), ("dq", q), ("dk", k), ("dv", v), ("tol_dq", q), ("tol_dk", k), ("tol_dv", v))}
    out["lse"] = torch.full((hq, T), -math.inf, dtype=torch.float64, device="cuda")
    out["tol_lse"] = torch.zeros((hq, T), dtype=torch.float64, device="cuda")
    for h in range(hq):
        Q, K, V = q[:, h].double(), k[:, h // per].double(), v[:, h // per].double()
        z = scale * Q @ K.t()
        size = scale * Q.abs() @ K.abs().t()
        bend = torch.ones_like(z)
        err = 2.0 ** -16 * size
        if m["cap"]:
            t = torch.tanh(z / m["cap"])
            z, bend = m["cap"] * t, 1 - t * t
            err = err + 2.0 ** -20 * m["cap"]
        if m["slopes"] is not None:
            z = z - m["slopes"][h].double() * far
            # log2 e (half a step), times the slope, times the distance, to the tile's column, to the
            # score, less the reference: 5.5 of 2^-24
            err = err + 2.0 ** -21 * m["slopes"][h].double().abs() * far
        err = (err * seen).amax(-1, keepdim=True) + 2.0 ** -20
        z = z.masked_fill(~seen, -math.inf)
        lse = torch.logsumexp(z, -1)
        p = torch.where(seen, (z - lse[:, None]).exp(), 0.0)
        o = p @ V
        out["o"][:, h], out["lse"][h] = o, lse
        lost = FLUSH * seen.double()
        out["tol_o"][:, h] = (STEP + 2 * err) * (p @ V.abs()) + STEP * o.abs() + lost @ V.abs()
        out["tol_lse"][h] = err[:, 0] + 2.0 ** -21 * (1 + torch.where(seen.any(-1), lse.abs(), 0.0))
        if not grads:
            continue
        dO = s["do"][:, h].double()
        dp = torch.where(seen, dO @ V.t(), 0.0)
        delta = (p * dp).sum(-1, keepdim=True)
        ds = p * (dp - delta) * bend
        # errors: of p (err), of dp's fp32 sum, of delta (from o as it is stored, but for rows of few
        # keys), of the operands' rounding to bf16
        e_dp = 2.0 ** -16 * (dO.abs() @ V.abs().t())
        e_delta = (STEP + 2 * err) * (dO.abs() * (p @ V.abs())).sum(-1, keepdim=True) + STEP * (dO.abs() * o.abs()).sum(-1, keepdim=True)
        e_ds = p * (e_dp + e_delta) + (2 * err + STEP + 2.0 ** -20) * p * (dp.abs() + delta.abs()) + STEP * ds.abs()
        e_ds = e_ds + lost * (1 + dp.abs() + delta.abs())
        e_p = (STEP + 2 * err) * p + lost
        out["dq"][:, h] = scale * ds @ K
        out["tol_dq"][:, h] = scale * e_ds @ K.abs() + STEP * out["dq"][:, h].abs()
        out["dk"][:, h // per] += scale * ds.t() @ Q
        out["tol_dk"][:, h // per] += scale * e_ds.t() @ Q.abs()
        out["dv"][:, h // per] += p.t() @ dO
        out["tol_dv"][:, h // per] += e_p.t() @ dO.abs()
    for n in ("dk", "dv"):
        out["tol_" + n] += STEP * out[n].abs()
    return out


def _near(got, ref, name):
    want, tol = ref[name], ref["tol_" + name]
    fine = torch.isfinite(want)
    assert got.shape == want.shape and torch.equal(torch.isfinite(got), fine), name
    over = ((got.double() - want).abs() - tol)[fine]
    assert not over.numel() or float(over.max()) <= 0, (name, float(over.max()), float((got.double() - want).abs()[fine].max()))


def _forward(s):
    st = B.new_status()
    o, lse = B.olive_packed_attention_fwd(s["q"], s["k"], s["v"], s["cu"], **s["more"], dev_status=st)
    assert B.status_bits(st) == []
    return o, lse


def _backward(s, o, lse, **kw):
    st = B.new_status()
    got = B.olive_packed_attention_bwd(s["do"], s["q"], s["k"], s["v"], o, lse, s["cu"], **s["more"], dev_status=st, **kw)
    assert B.status_bits(st) == []
    return got


def _check(s):
    ref = _reference(s, True)
    o, lse = _forward(s)
    _near(o, ref, "o")
    _near(lse, ref, "lse")
    behind = int(s["cu"][-1])
    assert not o[behind:].any() and bool((lse[:, behind:] == -math.inf).all())
    grads = _backward(s, o, lse)
    for name, g in zip(("dq", "dk", "dv"), grads):
        _near(g, ref, name)
        assert not g[behind:].any(), name
    return (o, lse, *grads)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 100, 127, 128, 129, 255, 256, 257, 300, 513, 1000])
@pytest.mark.parametrize("hq,hk,D", [(2, 1, 128), (3, 1, 64)])
def test_lengths(n, hq, hk, D):
    _check(_case([n], hq, hk, D, seed=n))


@pytest.mark.parametrize("D", [8, 16, 24, 32, 56, 64, 72, 80, 96, 104, 120, 128])
@pytest.mark.parametrize("hq,hk", [(1, 1), (4, 2)])
def test_widths(D, hq, hk):
    _check(_case([77, 200], hq, hk, D, seed=D))


@pytest.mark.parametrize("hq,hk", [(1, 1), (2, 2), (2, 1), (8, 2), (5, 1), (9, 3), (12, 12), (40, 8)])
@pytest.mark.parametrize("causal", [True, False])
def test_heads(hq, hk, causal):
    _check(_case([130, 7, 300], hq, hk, 64, causal=causal, seed=hq))


FORMS = [dict(), dict(causal=False), dict(prefix=50), dict(prefix=0), dict(prefix=1), dict(prefix=200), dict(cap=5.0), dict(bias=True),
         dict(cap=2.0, bias=True, prefix=140), dict(causal=False, bias=True), dict(scale=0.7), dict(sharp=4.0), dict(sharp=4.0, cap=30.0)]


@pytest.mark.parametrize("form", FORMS, ids=str)
@pytest.mark.parametrize("hq,hk,D", [(4, 2, 128), (3, 3, 40)])
def test_forms(form, hq, hk, D):
    _check(_case([1, 300, 129, 0, 17, 128, 2, 400], hq, hk, D, pad=33, **form))


def test_many_sequences():
    """More than a warp looks for at once, empty and single ones among them."""
    gen = torch.Generator().manual_seed(0)
    lens = torch.randint(0, 5, (1200,), generator=gen).tolist()
    lens[700] = 150
    _check(_case(lens, 2, 1, 32))
    _check(_case(lens, 3, 1, 32, causal=False, pad=5))


def test_largest_scores_late():
    """Each tile's keys outweigh those before them: the reference has to follow."""
    s = _case([700], 2, 1, 64)
    by = torch.linspace(0.2, 12, 700, device="cuda")[:, None, None]
    s["k"].copy_((s["q"][:, :1].float().mean(0, keepdim=True) * 0 + 1) * by.to(BF16))
    s["q"].copy_(s["q"].abs())
    _check(s)


def test_largest_scores_early():
    """The same the other way round."""
    s = _case([700], 2, 1, 64)
    by = torch.linspace(12, 0.2, 700, device="cuda")[:, None, None]
    s["k"].copy_(torch.ones_like(s["k"]) * by.to(BF16))
    s["q"].copy_(s["q"].abs())
    _check(s)


@pytest.mark.parametrize("slope", [-0.5, -0.03, 0.03, 0.5, 4.0])
@pytest.mark.parametrize("form", [dict(), dict(prefix=300), dict(causal=False), dict(cap=5.0)], ids=str)
def test_slopes(form, slope):
    """Scores that fall, or rise, with the distance by up to 500 a tile."""
    s = _case([700, 129, 1], 2, 1, 64, bias=True, **form)
    s["more"]["slopes"] = torch.tensor([slope, slope / 3], device="cuda")
    _check(s)


@pytest.mark.parametrize("form", [dict(), dict(cap=6.0), dict(cap=3.0, bias=True, prefix=20), dict(causal=False)], ids=str)
def test_what_is_not_finite(form):
    """A bad token behind a sequence's end, or in another one, does not show, not in a bit; its own
    sequence's does."""
    s = _case([100, 77, 60], 4, 2, 64, pad=20, **form)
    good = _check(s)
    for n in ("q", "k", "v", "do"):
        s[n][100 + 77:] = float("nan")  # the last sequence, and nobody's rows
    o, lse = _forward(s)
    assert torch.equal(o[:177], good[0][:177]) and torch.equal(lse[:, :177], good[1][:, :177])
    for g, want in zip((o, *_backward(s, o, lse)), (good[0], *good[2:])):
        assert torch.equal(g[:177], want[:177]) and torch.isnan(g[177:237]).all() and not g[237:].any()


@pytest.mark.parametrize("form", [dict(cap=20.0), dict(cap=5.0, bias=True), dict(prefix=900), dict(causal=False, cap=20.0)], ids=str)
def test_the_same_bits_whatever_ran_before(form):
    """What earlier launches left in shared and tensor memory decides nothing."""
    s = _case([2000, 45, 130], 5, 1, 128, **form)
    other = _case([700] * 3, 5, 1, 128, sharp=8.0, seed=1)
    run = lambda: (lambda o, lse: (o, lse, *_backward(s, o, lse)))(*_forward(s))
    want = run()
    for _ in range(8):
        _backward(other, *_forward(other))
        assert all(torch.equal(a, b) for a, b in zip(run(), want))


def test_layouts():
    """The same values in other layouts give the same bits."""
    s = _case([200, 61], 4, 2, 80, pad=3)
    want = _check(s)
    for lay in ("heads first", "wide"):
        def relaid(t):
            if lay == "heads first":
                return t.transpose(0, 1).contiguous().transpose(0, 1)
            wide = torch.full((t.shape[0], t.shape[1] + 3, t.shape[2] + 16), float("nan"), dtype=BF16, device="cuda")
            wide[:, 1:-2, 8:-8] = t
            return wide[:, 1:-2, 8:-8]
        q, k, v, do = (relaid(s[n]) for n in ("q", "k", "v", "do"))
        out = relaid(torch.zeros_like(want[0]))
        o, lse = B.olive_packed_attention_fwd(q, k, v, s["cu"], **s["more"], out=out)
        outs = [relaid(torch.zeros_like(t)) for t in want[2:]]
        grads = B.olive_packed_attention_bwd(do, q, k, v, o, lse, s["cu"], **s["more"], out=outs)
        assert o is out and all(a is b for a, b in zip(grads, outs))
        assert all(torch.equal(a, b) for a, b in zip((o, lse, *grads), want))
    # key heads that share memory
    one = s["k"][:, :1].contiguous()
    res = []
    for kv in (one.expand(-1, 2, -1), one.repeat(1, 2, 1)):
        o, lse = B.olive_packed_attention_fwd(s["q"], kv, kv, s["cu"], **s["more"])
        res.append((o, lse, *B.olive_packed_attention_bwd(s["do"], s["q"], kv, kv, o, lse, s["cu"], **s["more"])))
    assert all(torch.equal(a, b) for a, b in zip(*res))


def test_rows_of_one_key_have_no_gradient_of_their_score():
    """A softmax of one key is constant: exactly zero."""
    for lens, kw in (([1] * 300, {}), ([1, 1, 1], dict(causal=False)), ([1] * 20, dict(cap=3.0, bias=True, prefix=1))):
        s = _case(lens, 4, 2, 64, **kw)
        _, _, dq, dk, dv = _check(s)
        assert not dq.any() and not dk.any() and bool(dv.any())


def test_gradient_against_differences():
    """Along a random direction, against central differences of the 64-bit forward (their truncation
    is below 1e-5 of the slope's terms; the gradients' operands are rounded to 2^-8)."""
    s = _case([90, 40], 4, 2, 64, cap=8.0, bias=True, prefix=30)
    o, lse = _forward(s)
    grads = _backward(s, o, lse)
    gen = torch.Generator(device="cuda").manual_seed(1)
    dirs = [torch.randn(s[n].shape, generator=gen, device="cuda", dtype=torch.float64) for n in "qkv"]
    e = 1e-3
    values = []
    for step in (e, -e):
        moved = {**s, **{n: s[n].double() + step * u for n, u in zip("qkv", dirs)}}
        values.append(float((_reference(moved)["o"] * s["do"].double()).sum()))
    slope = (values[0] - values[1]) / (2 * e)
    terms = [g.double() * u for g, u in zip(grads, dirs)]
    got, size = sum(float(t.sum()) for t in terms), sum(float(t.abs().sum()) for t in terms)
    assert abs(got - slope) <= 3 * STEP * size


def test_autograd_form():
    s = _case([90, 33], 4, 2, 64, pad=5, prefix=10, cap=9.0, bias=True)
    leaves = [s[n].clone().requires_grad_() for n in "qkv"]
    o = B.packed_attention(*leaves, s["cu"], **s["more"])
    (torch.cat([o, o], 1)[:, 2:6].float() * s["do"].float()).sum().backward()
    o2, lse = _forward(s)
    s["do"] = torch.cat([s["do"][:, 2:], s["do"][:, :2]], 1)
    assert torch.equal(o, o2) and all(torch.equal(t.grad, g) for t, g in zip(leaves, _backward(s, o2, lse)))
    for loss in (lambda o: o.sum(), lambda o: (o * o.new_ones(1, 4, 64)).sum()):  # gradients that are one row for all
        got = torch.autograd.grad(loss(B.packed_attention(*leaves, s["cu"], **s["more"])), leaves)
        s["do"] = torch.ones_like(o2)
        assert all(torch.equal(a, b) for a, b in zip(got, _backward(s, o2, lse)))
    g, = torch.autograd.grad(B.packed_attention(*leaves, s["cu"]).square().sum(), leaves[0], create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g.sum(), leaves[0])


def test_captured_and_on_another_stream():
    s = _case([700, 45, 300], 8, 2, 128, pad=9)

    def run():
        o, lse = B.olive_packed_attention_fwd(s["q"], s["k"], s["v"], s["cu"], **s["more"])
        return (o, lse, *B.olive_packed_attention_bwd(s["do"], s["q"], s["k"], s["v"], o, lse, s["cu"], **s["more"]))

    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run()
    both = run()  # beside it
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) and torch.equal(c, b) for a, b, c in zip(got, want, both))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for seed, lens in ((5, [1, 1000, 44]), (6, [500, 545, 0])):  # (other sequences in the same arrays)
        new = _case(lens, 8, 2, 128, pad=9, seed=seed)
        for n in ("q", "k", "v", "do", "cu"):
            s[n].copy_(new[n])
        want = run()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("cu", [[0, 50, 40, 90], [0, 200], [5, 50], [-3, 60], [0, 2**31 - 1], [70, 20]])
def test_offsets_that_do_not_describe_the_batch(cu):
    s = _case([100], 2, 1, 64)
    st = B.new_status()
    bad = torch.tensor(cu, dtype=torch.int32, device="cuda")
    B.olive_packed_attention_fwd(s["q"], s["k"], s["v"], bad, dev_status=st)
    o, lse = B.olive_packed_attention_fwd(s["q"], s["k"], s["v"], bad)
    assert B.status_bits(st) == ["OLIVE_ERR_OFFSETS"]
    st = B.new_status()
    B.olive_packed_attention_bwd(s["do"], s["q"], s["k"], s["v"], o, lse, bad, dev_status=st)
    assert B.status_bits(st) == ["OLIVE_ERR_OFFSETS"]


@pytest.mark.parametrize("causal", [True, False])
def test_sequences_without_tokens(causal):
    """All of them: every row is behind the last one, whatever it holds."""
    s = _case([0, 0, 0], 3, 1, 64, pad=300, causal=causal)
    for n in ("q", "k", "v", "do"):
        s[n].fill_(float("nan"))
    o, lse = _forward(s)
    assert not o.any() and bool((lse == -math.inf).all())
    assert not any(g.any() for g in _backward(s, o, lse))


@pytest.mark.parametrize("n", [15, 16, 17, 18, 33])
@pytest.mark.parametrize("form", [dict(), dict(prefix=16), dict(prefix=17), dict(causal=False), dict(cap=4.0, bias=True)], ids=str)
@pytest.mark.parametrize("D", [8, 24, 128])
def test_rows_of_few_keys(n, form, D):
    """Around the number of keys up to which a row's delta comes from the keys."""
    _check(_case([n, 1, n - 1, 2], 6, 2, D, sharp=2.0, pad=3, **form))


def test_outputs_beside_others():
    """Gradients written into views of one array leave what lies between them."""
    s = _case([100, 60], 4, 2, 64, pad=7)
    o, lse = _forward(s)
    want = _backward(s, o, lse)
    wide = torch.full((167, 4 + 2 + 2 + 3, 64), 7.0, dtype=BF16, device="cuda")
    got = _backward(s, o, lse, out=(wide[:, :4], wide[:, 5:7], wide[:, 8:10]))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert bool((wide[:, [4, 7, 10]] == 7).all())


def test_no_tokens():
    s = _case([1], 2, 1, 64)
    o, lse = B.olive_packed_attention_fwd(s["q"][:0], s["k"][:0], s["v"][:0], torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert o.shape == (0, 2, 64) and lse.shape == (2, 0)
    got = B.olive_packed_attention_bwd(o, s["q"][:0], s["k"][:0], s["v"][:0], o, lse, torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert [tuple(t.shape) for t in got] == [(0, 2, 64), (0, 1, 64), (0, 1, 64)]
    s = _case([0, 0], 2, 1, 64, pad=10)
    _check(s)
