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
