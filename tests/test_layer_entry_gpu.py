"""The layer's autograd forms and clip_grad_norm_ on what autograd and a model hand to them."""

import pytest
import torch

from paper_2609_36246_gb300 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("limit", [0.3, 1e6])
def test_gradients_of_any_layout_are_clipped(dtype, limit):
    """As contiguous ones of the same values are (the norm's sums, and so its last bits, go by the
    order of the values in memory: 1e-6 of it; a value's own rounding is half a last place)."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    draw = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(dtype)
    grads = [draw(40, 30).t(), draw(30, 80)[:, ::2], draw(7, 5, 9).permute(1, 2, 0), draw(33), draw(50, 1).expand(50, 1),
             draw(3, 4, 6)[:, 1:3]]
    params = [torch.nn.Parameter(torch.zeros(g.shape, dtype=dtype, device="cuda")) for g in grads]
    before = [g.double() for g in grads]
    for p, g in zip(params, grads):
        p.grad = g
    norm = float(sum(b.square().sum() for b in before)) ** 0.5
    f = min(1.0, limit / (norm + 1e-6))
    got = float(B.clip_grad_norm_(params, limit))
    assert abs(got - norm) <= 1e-6 * norm
    tol = 2.0 ** -8 * 1.01 if dtype == torch.bfloat16 else 2e-6
    for p, g, b in zip(params, grads, before):
        assert p.grad is g and ((g.double() - b * f).abs() <= tol * (b * f).abs() + 1e-40).all()
        if limit == 1e6:
            assert torch.equal(g.double(), b)


def test_autograd_forms_report_what_the_device_found(monkeypatch):
    """A wait that ran out (there is no time to wait) and a position outside the tables."""
    draw = lambda *s: torch.randn(*s, device="cuda").to(torch.bfloat16)
    mlp = [t.requires_grad_() for t in (draw(900, 32768), *(draw(1024, 32768) * 0.005 for _ in range(2)), draw(32768, 1024))]
    before, after = B.new_status(), B.new_status()
    monkeypatch.setenv("OLIVE_WAIT_LIMIT_MS", "0")
    B.gated_mlp(*mlp, dev_status=before)
    monkeypatch.delenv("OLIVE_WAIT_LIMIT_MS")
    y = B.gated_mlp(*mlp, dev_status=after)
    assert B.status_bits(before) == ["OLIVE_ERR_TIMEOUT"] and B.status_bits(after) == []
    monkeypatch.setenv("OLIVE_WAIT_LIMIT_MS", "0")
    y.backward(torch.ones_like(y))
    torch.cuda.synchronize()
    monkeypatch.delenv("OLIVE_WAIT_LIMIT_MS")
    assert B.status_bits(after) == ["OLIVE_ERR_TIMEOUT"]

    q, k, w = draw(5, 3, 64).requires_grad_(), draw(5, 2, 64), draw(64)
    table = torch.ones(4, 32, device="cuda")
    for wrong in (False, True):
        pos = torch.tensor([0, 1, 2, 3, 4 if wrong else 0], dtype=torch.int32, device="cuda")
        st = B.new_status()
        yq, _ = B.qk_norm_rope(q, k, w, w, table, table, pos, dev_status=st)
        bits = ["OLIVE_ERR_TOKEN_RANGE"] if wrong else []
        assert B.status_bits(st) == bits
        st.zero_()
        yq.backward(torch.ones_like(yq))
        assert B.status_bits(st) == bits


def test_a_step_of_the_example_reports_too(monkeypatch):
    from examples import student_layer_step as E

    batch, T = E.draw_batch(512, [(20, 40), (9, 60)])
    p = E.init(512, 64, 2, 1, 32, 136)
    for rows, bits in ((128, []), (64, ["OLIVE_ERR_TOKEN_RANGE"])):  # the second sequence has 69 tokens
        st = B.new_status()
        E.step(p, batch, 512, T, 2, 1, E.rope_tables(rows, 32), dev_status=st)
        assert B.status_bits(st) == bits


@pytest.mark.parametrize("T", [16, 700])
def test_scoring_with_parameters_saves_nothing(T):
    """Under no_grad a call holds what olive_gated_mlp_fwd holds without saving, and gives its bits."""
    draw = lambda *s: torch.randn(*s, device="cuda").to(torch.bfloat16)
    x, w = draw(T, 256), [torch.nn.Parameter(t) for t in (draw(4096, 256), draw(4096, 256), draw(256, 4096))]

    def peak(f):
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        start = torch.cuda.memory_allocated()
        y = f()
        return torch.cuda.max_memory_allocated() - start, y

    want, y = peak(lambda: B.olive_gated_mlp_fwd(x, *w)[0])
    with torch.no_grad():
        got, z = peak(lambda: B.gated_mlp(x, *w))
    assert got <= want and torch.equal(y, z)
    assert peak(lambda: B.gated_mlp(x, *w))[0] >= want + 4 * T * 4096


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [8, 64])
@pytest.mark.parametrize("before,after", [(0, 4), (4, 0), (3, 1), (8, 8)])
def test_heads_inside_a_wider_tensor(dtype, D, before, after):
    """The gradients of heads that go on beside other columns have the bits of contiguous ones."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    draw = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(dtype)
    T, w = 21, [draw(D), draw(D)]
    table = [draw(T, 4).float(), draw(T, 4).float()]
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    heads = [draw(T, 3, D), draw(T, 2, D)]
    weigh = [draw(T, h.shape[1], before + D + after) for h in heads]
    leaf = [h.clone().requires_grad_() for h in heads]
    total = 0
    for y, g in zip(B.qk_norm_rope(*leaf, *w, *table, pos), weigh):
        wide = torch.cat([g[..., :before], y, g[..., before + D:]], -1)
        total = total + (wide.float() * g.float()).sum()
    total.backward()
    own = [g[..., before:before + D].contiguous() for g in weigh]
    want = B.olive_qk_norm_rope_bwd(*own, *heads, *w, *table, pos)
    assert all(torch.equal(t.grad, d) for t, d in zip(leaf, want))


def test_block_output_gradient_that_starts_anywhere():
    draw = lambda *s: torch.randn(*s, device="cuda").to(torch.bfloat16)
    x, w, flat = draw(70, 64), (draw(72, 64), draw(72, 64), draw(64, 72)), draw(70 * 64 + 3)
    dy = flat[3:].view(70, 64)
    leaf = x.clone().requires_grad_()
    B.gated_mlp(leaf, *w).backward(dy)
    _, saved = B.olive_gated_mlp_fwd(x, *w, save=True)
    want = B.olive_gated_mlp_bwd(dy.clone(), x, *w, saved, need_dW=False)[0]
    assert torch.equal(leaf.grad, want)
