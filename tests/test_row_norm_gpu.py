"""Rows' norm against the definition in 64 bits.

Tolerances.  Sums over a row are fp32: a thread adds up to 32 values, then up to 9 pairs and 16
warps, so a mean is off by at most 57 2^-24 < 2^-18 of the mean of its terms' magnitudes, and so is r
(half of the mean square's error, and a rounding or two).  With N = |n| + r mean|h| (the second term:
what the mean's error makes of n) a normalised value is within 2^-16 of N, and the gradient's three
terms within 2^-15 of theirs.  Rounding to the type adds half a last place, 2^-8 or 2^-24 of the
value.  The weights' gradients: a thread adds up to T / blocks rows (at most 30 here) in fp32.
"""

import pytest
import torch

from paper_2609_36246_gb300 import binding as B

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-5
WIDTHS = [8, 16, 248, 256, 264, 512, 520, 1000, 1024, 1032, 2040, 2048, 2056, 4096, 4104, 8192, 8200, 16384]


def _case(T, d, dtype, seed=0, offset=0.3, bias=True, residual=False):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    s = dict(x=(r(T, d) * (0.2 + 3 * torch.rand(T, 1, generator=gen, device="cuda")) + offset * r(T, 1)).to(dtype),
             w=(1 + 0.3 * r(d)).to(dtype), b=(0.3 * r(d)).to(dtype) if bias else None, dy=r(T, d).to(dtype),
             residual=r(T, d).to(dtype) if residual else None, g_h=r(T, d).to(dtype) if residual else None)
    return s


def _reference(s, h, kind):
    """y, dx, dw, db in 64 bits for the rows h, and what bounds their errors."""
    h = h.double()
    w, dy = s["w"].double(), s["dy"].double()
    b = torch.zeros_like(w) if s["b"] is None else s["b"].double()
    m = h.mean(-1, keepdim=True) if kind == "layer" else 0 * h[:, :1]
    r = 1 / ((h - m).square().mean(-1, keepdim=True) + EPS).sqrt()
    n = (h - m) * r
    N = n.abs() + (r * h.abs().mean(-1, keepdim=True) if kind == "layer" else 0)
    a = dy * w
    dx = a - n * (a * n).mean(-1, keepdim=True) - (a.mean(-1, keepdim=True) if kind == "layer" else 0)
    dx = r * dx + (0 if s["g_h"] is None else s["g_h"].double())
    A = a.abs()
    return dict(y=(n * w + b, 2.0 ** -16 * (w.abs() * N + b.abs())),
                dx=(dx, 2.0 ** -15 * r * (A + A.mean(-1, keepdim=True) + N * (A * N).mean(-1, keepdim=True)) +
                    2.0 ** -22 * (0 if s["g_h"] is None else s["g_h"].double().abs())),
                dw=((dy * n).sum(0), 2.0 ** -15 * (dy.abs() * N).sum(0)), db=(dy.sum(0), 2.0 ** -15 * dy.abs().sum(0)))


def _near(got, ref, what):
    want, slack = ref
    assert got.shape == want.shape, what
    over = (got.double() - want).abs() - slack - torch.finfo(got.dtype).eps / 2 * 1.01 * want.abs()
    assert not over.numel() or float(over.max()) <= 0, (what, float(over.max()))


def _check(s, kind):
    y, h, stats = B.olive_row_norm_fwd(s["x"], s["w"], s["b"], s["residual"], EPS, kind, save=True)
    if s["residual"] is None:
        assert h is s["x"]
    else:
        assert torch.equal(h, (s["x"].float() + s["residual"].float()).to(h.dtype))
    dx, dw, db = B.olive_row_norm_bwd(s["dy"], h, s["w"], stats, s["g_h"], kind, need_db=s["b"] is not None)
    ref = _reference(s, h, kind)
    for name, t in (("y", y), ("dx", dx), ("dw", dw), ("db", db)):
        if t is not None:
            assert t.dtype == (s["x"].dtype if name in ("y", "dx") else F32)
            _near(t, ref[name], name)
    return y, dx, dw, db


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("d", WIDTHS)
def test_widths(d, kind, dtype):
    _check(_case(37, d, dtype), kind)


@pytest.mark.parametrize("T", [1, 2, 3, 5, 127, 1001, 9000])
@pytest.mark.parametrize("dtype,residual,bias", [(BF16, True, True), (F32, True, False), (BF16, False, False)])
def test_rows(T, dtype, residual, bias):
    _check(_case(T, 520, dtype, T, residual=residual, bias=bias), "layer")
    _check(_case(T, 128, dtype, T, residual=residual, bias=bias), "rms")


def test_rows_far_from_zero():
    """A mean a thousand times the deviation: the deviation comes from the differences."""
    s = _case(64, 4096, F32)
    s["x"] = (s["x"] + 3000).contiguous()
    _check(s, "layer")


def test_rows_of_zeros_huge_and_bad_values():
    s = _case(6, 1000, F32)
    s["x"][0] = 0
    s["x"][1] *= 1e15
    s["x"][2] *= 1e-15
    _check(s, "layer")
    y, _, _ = B.olive_row_norm_fwd(s["x"], s["w"], s["b"], eps=EPS)
    assert torch.equal(y[0], s["b"])
    s["x"][3, 5], s["x"][4, 999] = float("nan"), float("inf")
    bad, _, _ = B.olive_row_norm_fwd(s["x"], s["w"], s["b"], eps=EPS)
    assert torch.isnan(bad[3]).all() and torch.isnan(bad[4]).all()
    keep = [0, 1, 2, 5]
    assert torch.equal(bad[keep], y[keep])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_outputs_in_place(dtype):
    s = _case(70, 2040, dtype, residual=True)
    y, h, stats = B.olive_row_norm_fwd(s["x"], s["w"], s["b"], s["residual"], EPS, save=True)
    x, res = s["x"].clone(), s["residual"].clone()
    y2, h2, stats2 = B.olive_row_norm_fwd(x, s["w"], s["b"], res, EPS, save=True, out=x, sum_out=res)
    assert y2 is x and h2 is res and torch.equal(y2, y) and torch.equal(h2, h) and torch.equal(stats2, stats)
    want = B.olive_row_norm_bwd(s["dy"], h, s["w"], stats, s["g_h"])
    for into in ("dy", "g_h"):
        t = dict(dy=s["dy"].clone(), g_h=s["g_h"].clone())
        got = B.olive_row_norm_bwd(t["dy"], h, s["w"], stats, t["g_h"], out=t[into])
        assert got[0] is t[into] and all(torch.equal(a, b) for a, b in zip(got, want))


def test_no_rows():
    s = _case(1, 64, BF16)
    none = s["x"][:0]
    y, _, stats = B.olive_row_norm_fwd(none, s["w"], s["b"], save=True)
    assert y.shape == (0, 64)
    dx, dw, db = B.olive_row_norm_bwd(none, none, s["w"], stats)
    assert dx.shape == (0, 64) and float(dw.abs().max()) == 0 and float(db.abs().max()) == 0


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_gradient_against_differences(kind):
    """Along a random direction, against central differences of the 64-bit forward (their truncation
    is below 1e-6 of the slope's terms; the gradients are within 2^-15 of theirs)."""
    s = _case(20, 264, F32, residual=True)
    y, h, stats = B.olive_row_norm_fwd(s["x"], s["w"], s["b"], s["residual"], EPS, kind, save=True)
    dx, dw, db = B.olive_row_norm_bwd(s["dy"], h, s["w"], stats, s["g_h"], kind)
    gen = torch.Generator(device="cuda").manual_seed(1)
    dirs = [torch.randn(t.shape, generator=gen, device="cuda", dtype=torch.float64) for t in (h, s["w"], s["b"])]

    def value(step):
        hh, w, b = (t.double() + step * u for t, u in zip((h, s["w"], s["b"]), dirs))
        m = hh.mean(-1, keepdim=True) if kind == "layer" else 0
        out = (hh - m) / ((hh - m).square().mean(-1, keepdim=True) + EPS).sqrt() * w + b
        return float((out * s["dy"].double()).sum() + (hh * s["g_h"].double()).sum())

    e = 1e-4
    slope = (value(e) - value(-e)) / (2 * e)
    terms = [g.double() * u for g, u in zip((dx, dw, db), dirs)]
    got, size = sum(float(t.sum()) for t in terms), sum(float(t.abs().sum()) for t in terms)
    assert abs(got - slope) <= 2.0 ** -14 * size


def test_autograd_form():
    s = _case(50, 520, BF16, residual=True)
    leaves = {k: s[k].clone().requires_grad_() for k in ("x", "w", "b", "residual")}
    y, h = B.row_norm(leaves["x"], leaves["w"], leaves["b"], leaves["residual"], EPS, "layer")
    # the sum is used too, and y's gradient comes as a view
    wide = torch.cat([y, y], 1)[:, 260:780]
    ((wide.float() * s["dy"].float()).sum() + (h.float() * s["g_h"].float()).sum()).backward()
    _, h0, stats = B.olive_row_norm_fwd(s["x"], s["w"], s["b"], s["residual"], EPS, save=True)
    dy = torch.cat([s["dy"][:, 260:], s["dy"][:, :260]], 1).contiguous()
    dx, dw, db = B.olive_row_norm_bwd(dy, h0, s["w"], stats, s["g_h"])
    for name, want in (("x", dx), ("residual", dx), ("w", dw.to(BF16)), ("b", db.to(BF16))):
        assert torch.equal(leaves[name].grad, want), name
    # only the sum, only y, and nothing kept where autograd is off
    x, w = leaves["x"], leaves["w"]
    x.grad = w.grad = None
    B.row_norm(x, w, None, leaves["residual"])[1].sum().backward()
    assert torch.equal(x.grad, torch.ones_like(x)) and w.grad is None
    y = B.row_norm(x, w, eps=EPS)
    g, = torch.autograd.grad(y.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g.sum(), x)
    with torch.no_grad():
        assert not B.row_norm(x, w).requires_grad and torch.equal(B.row_norm(x, w, eps=EPS), y)


def test_captured_and_on_another_stream():
    s = _case(700, 1032, BF16, residual=True)

    def run():
        y, h, stats = B.olive_row_norm_fwd(s["x"], s["w"], s["b"], s["residual"], EPS, save=True)
        return (y, h, *B.olive_row_norm_bwd(s["dy"], h, s["w"], stats, s["g_h"]))

    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for seed in (5, 6):
        for k, v in _case(700, 1032, BF16, seed, residual=True).items():
            s[k].copy_(v)
        want = run()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
