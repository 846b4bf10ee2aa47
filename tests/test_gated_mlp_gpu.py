"""Gated feed-forward block against its definition in 64 bits.

Tolerances.  bf16 holds 8 significant bits: one rounding is off by at most half a last place, 2^-8
of the value, and by less than 2^-8 / sqrt(3) in the mean square.  Forward: h is rounded as an
operand and y at the end; gradients: dg, du (or h) as operands, and the gradient at the end, unless
it stays in fp32.  Two such errors are independent, so in the norm they are below sqrt(2/3) 2^-8:
2^-8 is allowed (for fp32 gradients, with one rounding of rms 0.0017 and a little for the saved
pre-activations' 2^-10, 1.25 * 2^-9).  Element by element the bound is the sum of what every term of
the element's product may be off by, without cancellation (_bounds), and the result's own rounding.
"""

import pytest
import torch

from paper_2609_36246_gb300 import binding as B

pytestmark = pytest.mark.gpu

ROWS_RTOL = 2.0 ** -8
F32_RTOL = 1.25 * 2.0 ** -9


def _act(g, act):
    F = torch.nn.functional
    return F.silu(g) if act == "silu" else F.gelu(g, approximate="tanh")


def _case(T, d, f, seed=0, residual=True):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    bf = lambda t: t.to(torch.bfloat16)
    return dict(x=bf(r(T, d)), W_gate=bf(r(f, d) * (1.3 / d ** 0.5)), W_up=bf(r(f, d) * (1.3 / d ** 0.5)),
                W_down=bf(r(d, f) * 0.05), residual=bf(r(T, d)) if residual else None,
                dy=bf(r(T, d) * 0.1))


def _reference(s, act):
    x, wg, wu, wd = leaf = [s[k].double().requires_grad_() for k in ("x", "W_gate", "W_up", "W_down")]
    y = (_act(x @ wg.t(), act) * (x @ wu.t())) @ wd.t()
    if s["residual"] is not None:
        y = y + s["residual"].double()
    return y.detach(), torch.autograd.grad(y, leaf, s["dy"].double())


def _bounds(s, act):
    """What each element of y, dx, dW_gate, dW_up, dW_down may be off by before its own rounding: an
    operand's rounding (2^-8), the saved pre-activations' (2^-10, the activation's slope and the
    slope's slope times g being below 1.2), and fp32 sums (2^-15 of their terms' magnitudes)."""
    x, wg, wu, wd, dy = (s[k].double() for k in ("x", "W_gate", "W_up", "W_down", "dy"))
    g, u = x @ wg.t(), x @ wu.t()
    a, dh = _act(g, act), dy @ wd
    e_g, e_u = 2.0 ** -15 * (x.abs() @ wg.t().abs()), 2.0 ** -15 * (x.abs() @ wu.t().abs())
    e_dh = 2.0 ** -15 * (dy.abs() @ wd.abs())

    def e_h(e_g, e_u):
        return 2.0 ** -8 * (a * u).abs() + 1.2 * e_g * u.abs() + a.abs() * e_u

    y = e_h(e_g, e_u) @ wd.t().abs()
    e_g, e_u = e_g + 2.0 ** -10 * g.abs(), e_u + 2.0 ** -10 * u.abs()
    e_dg = (1.2 * 2.0 ** -8 + 2.0 ** -10) * (dh * u).abs() + 1.2 * (e_dh * u.abs() + dh.abs() * e_u + (dh * u).abs() * e_g)
    e_du = 2.0 ** -8 * (dh * a).abs() + e_dh * a.abs() + 1.2 * dh.abs() * e_g
    h = e_h(e_g, e_u)
    return (y, (e_dg @ wg.abs() + e_du @ wu.abs(), e_dg.t() @ x.abs(), e_du.t() @ x.abs(), dy.abs().t() @ h))


def _close(got, ref, rtol, what, bound=None):
    got, ref = got.double(), ref.double()
    assert got.shape == ref.shape and torch.isfinite(got).all(), what
    norm = ref.norm()
    if norm == 0:
        assert got.abs().max() == 0, what
        return
    rel = float((got - ref).norm() / norm)
    assert rel <= rtol, (what, rel)
    if bound is not None:
        over = (got - ref).abs() - (2.0 ** -8 * ref.abs() + 1.01 * bound + 1e-30)
        assert float(over.max()) <= 0, (what, float(over.max()), int(over.argmax()))


def _check(T, d, f, act="silu", residual=True, grad_dtype=torch.bfloat16, seed=0):
    s = _case(T, d, f, seed, residual)
    w = (s["W_gate"], s["W_up"], s["W_down"])
    st = B.new_status()
    y, saved = B.olive_gated_mlp_fwd(s["x"], *w, residual=s["residual"], act=act, save=True, dev_status=st)
    y2, none = B.olive_gated_mlp_fwd(s["x"], *w, residual=s["residual"], act=act, dev_status=st)
    got = B.olive_gated_mlp_bwd(s["dy"], s["x"], *w, saved, act=act, grad_dtype=grad_dtype, dev_status=st)
    assert none is None and B.status_bits(st) == []
    ref, grads = _reference(s, act)
    e_y, e_grads = _bounds(s, act)
    _close(y, ref, ROWS_RTOL, "y", e_y)
    assert torch.equal(y, y2)
    tol = ROWS_RTOL if grad_dtype == torch.bfloat16 else F32_RTOL
    for g, r, e, n in zip(got, grads, e_grads, ("dx", "dW_gate", "dW_up", "dW_down")):
        assert g.dtype == grad_dtype
        _close(g, r, tol, n, e)


@pytest.mark.parametrize("T", [1, 2, 7, 16, 17, 31, 33, 64, 65, 127, 128, 129, 255, 257, 511, 1000])
def test_rows(T):
    _check(T, 256, 704)


@pytest.mark.parametrize("d,f", [(8, 8), (64, 64), (72, 136), (128, 120), (264, 1000), (1000, 264), (2040, 600)])
@pytest.mark.parametrize("T", [1, 100, 300])
def test_odd_widths(T, d, f):
    _check(T, d, f, act="gelu_tanh", residual=T != 100)


@pytest.mark.parametrize("T,d,f", [(1, 4096, 1504), (40, 1536, 4104), (700, 2560, 2736), (2777, 1024, 2040)])
@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_larger(T, d, f, act):
    _check(T, d, f, act=act, grad_dtype=torch.float32 if act == "silu" else torch.bfloat16)


def test_rows_do_not_depend_on_the_batch_beside_them():
    """A NaN or an infinity in one row stays in that row of y and dx."""
    T, d, f, bad = 300, 128, 256, 131
    s = _case(T, d, f)
    w = (s["W_gate"], s["W_up"], s["W_down"])
    for value in (float("nan"), float("inf")):
        x = s["x"].clone()
        x[bad, 5] = value
        y, saved = B.olive_gated_mlp_fwd(x, *w, save=True)
        clean, saved0 = B.olive_gated_mlp_fwd(s["x"], *w, save=True)
        keep = torch.arange(T, device="cuda") != bad
        assert torch.equal(y[keep], clean[keep]) and not torch.isfinite(y[bad]).all()
        dx = B.olive_gated_mlp_bwd(s["dy"], x, *w, saved, need_dW=False)[0]
        dx0 = B.olive_gated_mlp_bwd(s["dy"], s["x"], *w, saved0, need_dW=False)[0]
        assert torch.equal(dx[keep], dx0[keep]) and not torch.isfinite(dx[bad]).all()


def test_few_rows_nan_stays_in_its_row():
    s = _case(9, 128, 256)
    w = (s["W_gate"], s["W_up"], s["W_down"])
    x = s["x"].clone()
    x[4, 100] = float("nan")
    y, _ = B.olive_gated_mlp_fwd(x, *w)
    clean, _ = B.olive_gated_mlp_fwd(s["x"], *w)
    keep = torch.arange(9, device="cuda") != 4
    assert torch.equal(y[keep], clean[keep]) and torch.isnan(y[4]).all()


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_extreme_preactivations(act):
    """Pre-activations of +-1e4 and of 1e-6: the activation's ends and its middle."""
    T, d, f = 64, 64, 128
    s = _case(T, d, f, residual=False)
    s["x"][:16] *= 1e4
    s["x"][16:32] *= 1e-6
    w = (s["W_gate"], s["W_up"], s["W_down"])
    y, saved = B.olive_gated_mlp_fwd(s["x"], *w, act=act, save=True)
    dx = B.olive_gated_mlp_bwd(s["dy"], s["x"], *w, saved, act=act, need_dW=False)[0]
    ref, grads = _reference(s, act)
    for rows in (slice(0, 16), slice(16, 32), slice(32, 64)):
        _close(y[rows], ref[rows], ROWS_RTOL, "y")
        _close(dx[rows], grads[0][rows], ROWS_RTOL, "dx")


def test_no_rows():
    s = _case(1, 64, 72)
    w = (s["W_gate"], s["W_up"], s["W_down"])
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    y, saved = B.olive_gated_mlp_fwd(x, *w, residual=x, save=True)
    assert y.shape == (0, 64) and saved.numel() == 0
    for dt in (torch.bfloat16, torch.float32):
        out = [torch.full(t.shape, 7.0, dtype=dt, device="cuda") for t in (x, *w)]
        B.olive_gated_mlp_bwd(x, x, *w, saved, grad_dtype=dt, out=out)
        assert all(float(g.abs().sum()) == 0 for g in out[1:])


def test_parts_of_the_backward_and_in_place_residual():
    s = _case(333, 256, 512)
    w = (s["W_gate"], s["W_up"], s["W_down"])
    y, saved = B.olive_gated_mlp_fwd(s["x"], *w, residual=s["residual"], save=True)
    r = s["residual"].clone()
    B.olive_gated_mlp_fwd(s["x"], *w, residual=r, out=r)
    assert torch.equal(r, y)
    whole = B.olive_gated_mlp_bwd(s["dy"], s["x"], *w, saved)
    dx = B.olive_gated_mlp_bwd(s["dy"], s["x"], *w, saved, need_dW=False)
    dW = B.olive_gated_mlp_bwd(s["dy"], s["x"], *w, saved, need_dx=False)
    assert dx[1:] == (None, None, None) and dW[0] is None
    # (the cut of the tiles, and with it the order of sums, is the launch's own)
    _close(dx[0], whole[0], ROWS_RTOL, "dx")
    for a, b in zip(dW[1:], whole[1:]):
        _close(a, b, ROWS_RTOL, "dW")


def test_same_call_same_bits_streams_and_graphs():
    for T, d, f in ((12, 2048, 768), (900, 1024, 1408)):
        s = _case(T, d, f)
        w = (s["W_gate"], s["W_up"], s["W_down"])

        def step():
            y, saved = B.olive_gated_mlp_fwd(s["x"], *w, residual=s["residual"], save=True)
            return (y, *B.olive_gated_mlp_bwd(s["dy"], s["x"], *w, saved))

        first = step()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(3):
                again = step()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, again))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured = step()
        for _ in range(3):
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, captured))


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_gradient_against_differences(act):
    """The gradients along a direction against central differences of the 64-bit forward.

    The step's truncation is below 1e-6 of the slope.  The gradients' errors are independent and at
    most 2^-8 of each element, so along a direction their sum is a few 2^-8 |grad * v|."""
    s = _case(70, 96, 200, residual=False)
    names = ("x", "W_gate", "W_up", "W_down")
    y, saved = B.olive_gated_mlp_fwd(*[s[k] for k in names], act=act, save=True)
    grads = B.olive_gated_mlp_bwd(s["dy"], *[s[k] for k in names], saved, act=act, grad_dtype=torch.float32)
    gen = torch.Generator(device="cuda").manual_seed(9)
    at = [s[k].double() for k in names]

    def loss(p):
        x, wg, wu, wd = p
        return float(((_act(x @ wg.t(), act) * (x @ wu.t())) @ wd.t() * s["dy"].double()).sum())

    for i, g in enumerate(grads):
        v = torch.randn(at[i].shape, generator=gen, device="cuda", dtype=torch.float64) * at[i].std()
        e = 1e-4
        moved = lambda t: loss([p + t * v if j == i else p for j, p in enumerate(at)])
        slope = (moved(e) - moved(-e)) / (2 * e)
        here = float((g.double() * v).sum())
        assert abs(here - slope) <= 6 * 2.0 ** -8 * float((g.double() * v).norm()) + 1e-6 * abs(slope), (i, here, slope)


def test_autograd():
    s = _case(150, 128, 256)
    leaf = [s[k].requires_grad_() for k in ("x", "W_gate", "W_up", "W_down", "residual")]
    B.gated_mlp(*leaf).backward(s["dy"])
    _, grads = _reference({k: v.detach() if v is not None else v for k, v in s.items()}, "silu")
    for t, r in zip(leaf, (*grads, s["dy"])):
        _close(t.grad, r, ROWS_RTOL, "grad")
    with torch.no_grad():
        assert not B.gated_mlp(*leaf).requires_grad


def test_refusals():
    s = _case(4, 64, 72)
    w = (s["W_gate"], s["W_up"], s["W_down"])
    with pytest.raises(TypeError):
        B.olive_gated_mlp_fwd(s["x"].float(), *w)
    with pytest.raises(TypeError):
        B.olive_gated_mlp_fwd(s["x"].t().contiguous().t(), *w)
    with pytest.raises(ValueError):
        B.olive_gated_mlp_fwd(s["x"], s["W_gate"], s["W_up"], s["W_up"])
    with pytest.raises(ValueError):
        B.olive_gated_mlp_fwd(s["x"], *w, residual=s["x"][:2])
    with pytest.raises(KeyError):
        B.olive_gated_mlp_fwd(s["x"], *w, act="relu")
    odd = [torch.zeros(*n, dtype=torch.bfloat16, device="cuda") for n in ((4, 60), (72, 60), (72, 60), (60, 72))]
    with pytest.raises(B.OliveError) as e:
        B.olive_gated_mlp_fwd(*odd)
    assert e.value.status == 3
    with pytest.raises(B.OliveError) as e:
        B.olive_gated_mlp_fwd(s["x"], *w, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 9


# shapes by the path they take: few rows with each count of tokens, by whole K steps and by clusters
# that share them (one token's tiles fill the GPU or do not); many rows in tiles of 128 and of 256
# columns, with every product whole, and with tiles cut in two and in many pieces
@pytest.mark.parametrize("T,d,f", [
    (5, 64, 20000), (5, 1000, 24), (20, 2048, 4096), (33, 512, 12288), (64, 4096, 512), (100, 136, 16384),
    (128, 2048, 2056), (128, 8, 4096), (3, 8, 8),
    (200, 1024, 2816), (512, 2048, 6144), (256, 4096, 1032), (130, 256, 8200), (1500, 4096, 264), (2000, 512, 4000),
    (9000, 64, 72), (4100, 1288, 1544)])
def test_paths(T, d, f):
    _check(T, d, f, act="gelu_tanh" if T % 2 else "silu", residual=T % 3 != 0,
           grad_dtype=torch.float32 if d % 16 else torch.bfloat16)


# both sides of the widths from which 65 to 128 rows take the weights as the wide operand, with the
# second product's K steps whole and shared by clusters
@pytest.mark.parametrize("T", [64, 65, 100, 128, 129])
@pytest.mark.parametrize("d,f", [(136, 4920), (136, 4928), (8, 4936), (1032, 5000), (2048, 4928)])
def test_wide_blocks(T, d, f):
    _check(T, d, f, act="gelu_tanh" if T % 2 else "silu", residual=T != 100,
           grad_dtype=torch.float32 if d == 136 else torch.bfloat16)


# the backward of few rows: each count of tokens, widths that end inside a block of 64 columns or
# just behind one, K steps whole and shared by clusters
@pytest.mark.parametrize("T", [1, 15, 16, 17, 32, 33, 63, 64, 65])
@pytest.mark.parametrize("d,f", [(8, 8), (56, 72), (64, 128), (136, 192), (200, 4104), (4104, 200), (1376, 3864)])
def test_few_rows_backward(T, d, f):
    _check(T, d, f, act="silu" if T % 2 else "gelu_tanh", grad_dtype=torch.float32 if T in (15, 33, 64) else torch.bfloat16)


@pytest.mark.parametrize("T", [1, 20, 64, 65])
@pytest.mark.parametrize("grad_dtype", [torch.bfloat16, torch.float32])
def test_parts_of_the_backward(T, grad_dtype):
    """dx alone and the weights' gradients alone, again and again: the same bits each time, on few rows
    those of the call for all (with more rows the products' sums are cut by what else is asked for),
    and right."""
    s = _case(T, 520, 1416)
    w = (s["W_gate"], s["W_up"], s["W_down"])
    y, saved = B.olive_gated_mlp_fwd(s["x"], *w, save=True)
    back = lambda **k: B.olive_gated_mlp_bwd(s["dy"], s["x"], *w, saved, grad_dtype=grad_dtype, **k)
    whole, dx, dw = back(), back(need_dW=False), back(need_dx=False)
    assert dx[1:] == (None, None, None) and dw[0] is None
    same = lambda a, b: all(torch.equal(g, h) for g, h in zip(a, b) if g is not None)
    for _ in range(5):
        assert same(back(need_dW=False), dx) and same(back(need_dx=False), dw) and same(back(), whole)
    if T <= 64:
        assert same(dx, whole) and same(dw, whole)
    _, ref = _reference(s, "silu")
    _, bounds = _bounds(s, "silu")
    tol = ROWS_RTOL if grad_dtype == torch.bfloat16 else F32_RTOL
    for g, r, e in zip((dx[0],) + dw[1:], ref, bounds):
        _close(g, r, tol, "part", e)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_few_rows_backward_keeps_a_bad_row_to_itself(bad):
    """A row of x or dy that is not finite leaves the other rows' dx as they were; its own is NaN."""
    T, d, f, at = 37, 136, 328, 18
    s = _case(T, d, f)
    w = (s["W_gate"], s["W_up"], s["W_down"])
    y, saved = B.olive_gated_mlp_fwd(s["x"], *w, save=True)
    want = B.olive_gated_mlp_bwd(s["dy"], s["x"], *w, saved, need_dW=False)[0]
    rest = [i for i in range(T) if i != at]
    for name in ("x", "dy"):
        t = {k: s[k].clone() for k in ("x", "dy")}
        t[name][at, 3] = bad
        y, saved = B.olive_gated_mlp_fwd(t["x"], *w, save=True)
        dx = B.olive_gated_mlp_bwd(t["dy"], t["x"], *w, saved, need_dW=False)[0]
        assert torch.equal(dx[rest], want[rest])
        assert not torch.isfinite(dx[at]).any()


@pytest.mark.parametrize("T,d,f", [(7, 131072, 512), (900, 32768, 1024)])
def test_waits_that_run_out_are_reported(T, d, f, monkeypatch):
    """With no time to wait the calls give up, say so and leave the context usable (the widths make
    the epilogues wait long enough for the limit to be looked at)."""
    s = _case(T, d, f)
    w = (s["W_gate"], s["W_up"], s["W_down"])
    y, saved = B.olive_gated_mlp_fwd(s["x"], *w, save=True)
    want = B.olive_gated_mlp_bwd(s["dy"], s["x"], *w, saved)
    monkeypatch.setenv("OLIVE_WAIT_LIMIT_MS", "0")
    for bwd in (False, True):
        st = B.new_status()
        if bwd:
            B.olive_gated_mlp_bwd(s["dy"], s["x"], *w, saved, dev_status=st)
        else:
            B.olive_gated_mlp_fwd(s["x"], *w, dev_status=st)
        torch.cuda.synchronize()
        assert B.status_bits(st) == ["OLIVE_ERR_TIMEOUT"]
    monkeypatch.delenv("OLIVE_WAIT_LIMIT_MS")
    st = B.new_status()
    again, saved2 = B.olive_gated_mlp_fwd(s["x"], *w, save=True, dev_status=st)
    got = B.olive_gated_mlp_bwd(s["dy"], s["x"], *w, saved2, dev_status=st)
    assert B.status_bits(st) == [] and torch.equal(again, y) and all(torch.equal(a, b) for a, b in zip(got, want))


def test_workspace_of_another_call_and_sticky_contents():
    """What an earlier call left in a workspace does not matter."""
    for T, d, f in ((30, 256, 512), (700, 512, 1544)):
        s = _case(T, d, f)
        w = (s["W_gate"], s["W_up"], s["W_down"])
        want, saved = B.olive_gated_mlp_fwd(s["x"], *w, save=True)
        grads = B.olive_gated_mlp_bwd(s["dy"], s["x"], *w, saved)
        for byte in (0x00, 0xff, 0x7f):
            ws = torch.full((B.olive_workspace_size("gated_mlp_bwd", T, d, f),), byte, dtype=torch.uint8, device="cuda")
            assert torch.equal(B.olive_gated_mlp_fwd(s["x"], *w, ws=ws)[0], want)
            ws.fill_(byte)
            got = B.olive_gated_mlp_bwd(s["dy"], s["x"], *w, saved, ws=ws)
            assert all(torch.equal(a, b) for a, b in zip(got, grads))
