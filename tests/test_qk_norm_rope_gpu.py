"""Heads' norm and rotation against the definition in 64 bits, and the packed positions.

Tolerances.  The kernels compute in fp32 and round once.  A rotated value is a sum of two terms of
at most the row's largest normalised value, each a few 2^-23 off, and r is off by the mean square's
error, at most D 2^-24 / 2 <= 2^-17 of it: 1e-5 of the row's largest value covers both.  bf16 adds
its rounding, half a last place: 2^-8 of the value (8 significant bits).  The weights' gradients are sums of T H terms of that accuracy; a
thread adds up to some hundred of them in fp32: 2^-15 of the sum of their magnitudes.
"""

import pytest
import torch

from paper_2609_36246_gb300 import binding as B

pytestmark = pytest.mark.gpu

EPS = 1e-6


def _tables(P, R, base=10000.0):
    a = torch.arange(P, device="cuda").double()[:, None] * base ** (-torch.arange(0, R, 2, device="cuda").double() / max(R, 1))
    return a.cos().float(), a.sin().float()


def _case(T, hq, hk, D, R, dtype, P=64, seed=0, fused=True):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    if fused:
        qkv = (r(T, hq + 2 * hk + 1, D) * (0.1 + torch.rand(T, hq + 2 * hk + 1, 1, generator=gen, device="cuda"))).to(dtype)
        q, k = qkv[:, :hq], qkv[:, hq:hq + hk]
    else:
        q, k = r(T, hq, D).to(dtype), r(T, hk, D).to(dtype)
    cos, sin = _tables(P, R)
    return dict(q=q, k=k, w_q=(1 + 0.3 * r(D)).to(dtype), w_k=(1 + 0.3 * r(D)).to(dtype), cos=cos, sin=sin,
                positions=torch.randint(0, P, (T,), generator=gen, device="cuda", dtype=torch.int32),
                g_q=r(T, hq, D).to(dtype), g_k=r(T, hk, D).to(dtype))


def _reference(s, inter):
    """Outputs, gradients and the weights' gradients with the sums of their terms' magnitudes."""
    R = 2 * s["cos"].shape[1]
    c, n = (s[k].double()[s["positions"].long()][:, None] for k in ("cos", "sin"))
    first = torch.arange(0, R, 2, device="cuda") if inter else torch.arange(R // 2, device="cuda")
    second = first + (1 if inter else R // 2)
    out = {}
    for side in ("q", "k"):
        x = s[side].double().detach().requires_grad_()
        w = s["w_" + side].double().requires_grad_()
        z = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
        v = z * w
        y = v.clone()
        y[..., first] = v[..., first] * c - v[..., second] * n
        y[..., second] = v[..., second] * c + v[..., first] * n
        out[side] = y.detach()
        g = s["g_" + side].double()
        if x.numel():
            out["d" + side], out["dw_" + side] = torch.autograd.grad(y, (x, w), g, retain_graph=True)
            dv, = torch.autograd.grad(y, v, g)
            out["sum_" + side] = (dv * z).abs().sum((0, 1)).detach()
            out["scale_" + side] = (dv * w).abs().amax(-1, keepdim=True) / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
        else:
            out["d" + side], out["dw_" + side] = torch.zeros_like(x), torch.zeros_like(w)
    return out


def _near(got, ref, scale, dtype, what):
    bound = 1e-5 * scale + (2.0 ** -8 * 1.01 * ref.abs() if dtype == torch.bfloat16 else 0)
    assert got.dtype == dtype and got.shape == ref.shape, what
    if got.numel():
        over = ((got.double() - ref).abs() - bound).max()
        assert float(over) <= 0, (what, float(over))


def _check(s, inter, dtype):
    st = B.new_status()
    more = (s["w_q"], s["w_k"], s["cos"], s["sin"], s["positions"], EPS, inter)
    yq, yk = B.olive_qk_norm_rope_fwd(s["q"], s["k"], *more, dev_status=st)
    dq, dk, dwq, dwk = B.olive_qk_norm_rope_bwd(s["g_q"], s["g_k"], s["q"], s["k"], *more, dev_status=st)
    assert B.status_bits(st) == []
    ref = _reference(s, inter)
    for side, y, d, dw in (("q", yq, dq, dwq), ("k", yk, dk, dwk)):
        top = ref[side].abs().amax(-1, keepdim=True) * 2 if y.numel() else 0
        _near(y, ref[side], top, dtype, side)
        # (a gradient is the difference of two terms of this size)
        _near(d, ref["d" + side], 2 * ref["scale_" + side].detach() if y.numel() else 0, dtype, "d" + side)
        assert dw.dtype == torch.float32
        if y.numel():
            assert ((dw.double() - ref["dw_" + side]).abs() <= 2.0 ** -15 * ref["sum_" + side]).all(), "dw_" + side
        else:
            assert float(dw.abs().max()) == 0
    return yq, yk, dq, dk, dwq, dwk


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,R", [(8, 8), (16, 8), (64, 64), (80, 80), (80, 32), (96, 48), (128, 128), (128, 0),
                                 (136, 136), (256, 256), (256, 64)])
def test_head_widths(D, R, inter, dtype):
    _check(_case(37, 6, 2, D, R, dtype), inter, dtype)


@pytest.mark.parametrize("T,hq,hk", [(1, 1, 1), (1, 32, 8), (2, 5, 0), (3, 0, 3), (100, 40, 8), (1001, 7, 1), (6000, 32, 8)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_tokens_and_heads(T, hq, hk, dtype):
    _check(_case(T, hq, hk, 128, 128, dtype), False, dtype)


@pytest.mark.parametrize("layout", ["contiguous", "heads first", "wide"])
def test_layouts(layout):
    """The same values in other layouts give the same bits, in and out."""
    dt = torch.bfloat16
    s = _case(50, 8, 4, 64, 64, dt, fused=False)
    want = _check(s, False, dt)
    more = (s["w_q"], s["w_k"], s["cos"], s["sin"], s["positions"], EPS, False)

    def relaid(t):
        if layout == "heads first":
            return t.transpose(0, 1).contiguous().transpose(0, 1)
        if layout == "wide":
            wide = torch.full((t.shape[0], t.shape[1] + 3, t.shape[2] + 16), float("nan"), dtype=dt, device="cuda")
            wide[:, 1:-2, 8:-8] = t
            return wide[:, 1:-2, 8:-8]
        return t.clone()

    q, k, gq, gk = (relaid(s[n]) for n in ("q", "k", "g_q", "g_k"))
    yq, yk = B.olive_qk_norm_rope_fwd(q, k, *more, out=(relaid(s["q"]), relaid(s["k"])))
    out = (relaid(s["q"]), relaid(s["k"]))
    got = (yq, yk, *B.olive_qk_norm_rope_bwd(gq, gk, q, k, *more, out=out))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_in_place():
    dt = torch.bfloat16
    s = _case(60, 8, 4, 128, 128, dt)
    more = (s["w_q"], s["w_k"], s["cos"], s["sin"], s["positions"], EPS, False)
    want = B.olive_qk_norm_rope_fwd(s["q"], s["k"], *more)
    wantd = B.olive_qk_norm_rope_bwd(s["g_q"], s["g_k"], s["q"], s["k"], *more)
    gq, gk = s["g_q"].clone(), s["g_k"].clone()
    got = B.olive_qk_norm_rope_bwd(gq, gk, s["q"], s["k"], *more, out=(gq, gk))
    assert all(torch.equal(a, b) for a, b in zip(got, wantd))
    B.olive_qk_norm_rope_fwd(s["q"], s["k"], *more, out=(s["q"], s["k"]))
    assert torch.equal(s["q"], want[0]) and torch.equal(s["k"], want[1])


def test_rows_of_zeros_and_of_huge_values():
    dt = torch.float32
    s = _case(4, 2, 1, 64, 64, dt, fused=False)
    s["q"][0] = 0
    s["q"][1] *= 1e15
    s["q"][2] *= 1e-12
    _check(s, False, dt)
    more = (s["w_q"], s["w_k"], s["cos"], s["sin"], s["positions"], EPS, False)
    yq, _ = B.olive_qk_norm_rope_fwd(s["q"], s["k"], *more)
    assert float(yq[0].abs().max()) == 0
    s["q"][1, 0, 3] = float("nan")
    bad, _ = B.olive_qk_norm_rope_fwd(s["q"], s["k"], *more)
    assert torch.isnan(bad[1, 0]).all()
    bad[1, 0], yq[1, 0] = 0, 0
    assert torch.equal(bad, yq)


@pytest.mark.parametrize("wrong", [-1, 64, 2**30])
def test_position_outside_the_tables(wrong):
    s = _case(20, 3, 2, 64, 32, torch.bfloat16)
    more = lambda: (s["w_q"], s["w_k"], s["cos"], s["sin"], s["positions"], EPS, False)
    want = B.olive_qk_norm_rope_fwd(s["q"], s["k"], *more())
    s["positions"] = s["positions"].clone()
    s["positions"][7] = wrong
    for bwd in (False, True):
        st = B.new_status()
        if bwd:
            got = B.olive_qk_norm_rope_bwd(s["g_q"], s["g_k"], s["q"], s["k"], *more(), dev_status=st)[:2]
        else:
            got = B.olive_qk_norm_rope_fwd(s["q"], s["k"], *more(), dev_status=st)
        assert B.status_bits(st) == ["OLIVE_ERR_TOKEN_RANGE"]
        for g in got:
            assert torch.isnan(g[7]).all()
        if not bwd:
            keep = torch.arange(20, device="cuda") != 7
            assert all(torch.equal(g[keep], w[keep]) for g, w in zip(got, want))


def test_no_tokens():
    s = _case(1, 3, 2, 64, 64, torch.bfloat16)
    for n in ("q", "k", "g_q", "g_k", "positions"):
        s[n] = s[n][:0]
    more = (s["w_q"], s["w_k"], s["cos"], s["sin"], s["positions"])
    yq, yk = B.olive_qk_norm_rope_fwd(s["q"], s["k"], *more)
    assert yq.shape == (0, 3, 64) and yk.shape == (0, 2, 64)
    got = B.olive_qk_norm_rope_bwd(s["g_q"], s["g_k"], s["q"], s["k"], *more)
    assert float(got[2].abs().max()) == 0 and float(got[3].abs().max()) == 0


def test_gradient_against_differences():
    """Along a random direction, against central differences of the 64-bit forward (truncation below
    1e-6 of the slope); the gradients are off by at most 1e-5 of their terms."""
    s = _case(40, 3, 2, 64, 48, torch.float32, fused=False)
    more = (s["w_q"], s["w_k"], s["cos"], s["sin"], s["positions"], EPS, True)
    dq, dk, dwq, dwk = B.olive_qk_norm_rope_bwd(s["g_q"], s["g_k"], s["q"], s["k"], *more)
    gen = torch.Generator(device="cuda").manual_seed(3)

    def loss(**change):
        r = _reference({**s, **change}, True)
        return float((r["q"] * s["g_q"].double()).sum() + (r["k"] * s["g_k"].double()).sum())

    for name, g in (("q", dq), ("k", dk), ("w_q", dwq), ("w_k", dwk)):
        v = torch.randn(s[name].shape, generator=gen, device="cuda", dtype=torch.float64)
        e = 1e-5
        slope = (loss(**{name: s[name].double() + e * v}) - loss(**{name: s[name].double() - e * v})) / (2 * e)
        assert abs(float((g.double() * v).sum()) - slope) <= 1e-5 * float((g.double() * v).abs().sum()), name


def test_streams_graphs_and_autograd():
    s = _case(500, 16, 4, 128, 128, torch.bfloat16)
    more = (s["w_q"], s["w_k"], s["cos"], s["sin"], s["positions"], EPS, False)
    step = lambda: (*B.olive_qk_norm_rope_fwd(s["q"], s["k"], *more),
                    *B.olive_qk_norm_rope_bwd(s["g_q"], s["g_k"], s["q"], s["k"], *more))
    first = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    graph.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(first, again, captured):
        assert torch.equal(a, b) and torch.equal(a, c)
    q, k = s["q"].detach().clone().requires_grad_(), s["k"].detach().clone().requires_grad_()
    wq, wk = s["w_q"].clone().requires_grad_(), s["w_k"].clone().requires_grad_()
    yq, yk = B.qk_norm_rope(q, k, wq, wk, *more[2:])
    torch.autograd.backward((yq, yk), (s["g_q"], s["g_k"]))
    for t, g in zip((q, k, wq, wk), first[2:]):
        assert torch.equal(t.grad, g.to(t.dtype))


@pytest.mark.parametrize("lens", [[1], [5, 1, 300], [0, 4, 0, 0, 7], [64] * 64])
def test_packed_positions(lens):
    cu = torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int32, device="cuda")
    want = torch.cat([torch.arange(n) for n in lens] + [torch.zeros(9, dtype=torch.int64)])
    got = B.olive_packed_positions(cu, sum(lens) + 9)
    assert got.dtype == torch.int32 and torch.equal(got.cpu().long(), want)


def test_refusals():
    s = _case(5, 3, 2, 64, 64, torch.bfloat16)
    args = lambda **kw: [{**s, **kw}[n] for n in ("q", "k", "w_q", "w_k", "cos", "sin", "positions")]
    f = B.olive_qk_norm_rope_fwd
    with pytest.raises(TypeError):
        f(*args(k=s["k"].float()))
    with pytest.raises(TypeError):
        f(*args(q=s["q"].transpose(1, 2).contiguous().transpose(1, 2)))
    with pytest.raises(TypeError):
        f(*args(positions=s["positions"].long()))
    with pytest.raises(ValueError):
        f(*args(positions=s["positions"][:3]))
    with pytest.raises(ValueError):
        f(*args(w_q=s["w_q"][:32]))
    for cos, sin, status in ((*_tables(8, 128), 2), (*_tables(8, 20), 3)):
        with pytest.raises(B.OliveError) as e:
            f(*args(cos=cos, sin=sin))
        assert e.value.status == status
    with pytest.raises(B.OliveError) as e:
        f(*args(), eps=-1.0)
    assert e.value.status == 1
    wide = torch.zeros(5, 3, 68, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B.OliveError) as e:
        f(*args(q=wide[..., 4:]))
    assert e.value.status == 3


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_values_that_are_not_finite_stay_where_the_formula_has_them(value, inter):
    """An infinite value makes its row's scale 0 and itself (and its pair's partner) NaN; a NaN takes
    the row.  Other rows do not change."""
    s = _case(6, 3, 1, 64, 32, torch.float32, fused=False)
    more = (s["w_q"], s["w_k"], s["cos"], s["sin"], s["positions"], EPS, inter)
    want, _ = B.olive_qk_norm_rope_fwd(s["q"], s["k"], *more)
    s["q"][2, 1, 40] = value
    got, _ = B.olive_qk_norm_rope_fwd(s["q"], s["k"], *more)
    keep = torch.ones(6, 3, dtype=torch.bool, device="cuda")
    keep[2, 1] = False
    assert torch.equal(got[keep], want[keep])
    bad = torch.isnan(got[2, 1])
    if value != value:
        assert bad.all()
    else:
        assert bad[40] and int(bad.sum()) == 1 and float(got[2, 1][~bad].abs().max()) == 0
