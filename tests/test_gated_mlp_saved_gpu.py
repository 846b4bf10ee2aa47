"""The 16-bit form in which the gated block saves its pre-activations, at the ends of its range.

Identity weights make a pre-activation a sum of two of x's values, exact in fp32, so what is saved has
to be the value rounded to nearest even at 10 significant bits, with steps of 2^-39 below 2^-30 and
2^33 - 2^24 in the place of anything larger; what is not finite is NaN.  The gradient that is formed
from it is rounded to bf16 as two operands and once at the end, each by at most half a place: 2 x 2^-8
of the terms' magnitudes together; the activation's own error (1e-6) is below a tenth of 2^-8 of them.
"""

import math

import pytest
import torch

from paper_2609_36246_gb300 import binding as B

pytestmark = pytest.mark.gpu

D = 64
TOP = 2.0 ** 33 - 2.0 ** 24


def _decode(bits):
    code = bits.cpu().to(torch.int64) & 0xffff
    e, f = (code >> 9) & 63, (code & 511).double()
    v = torch.where(e > 0, torch.ldexp(1 + f / 512, e - 31), f * 2.0 ** -39)
    v = torch.where((code & 0x7fff) == 0x7fff, torch.nan, v)
    return torch.where(code >= 0x8000, -v, v)


def _held(v):
    if not math.isfinite(v):
        return math.nan
    step = 2.0 ** (max(math.frexp(v)[1] - 1, -30) - 9)
    return math.copysign(min(abs(round(v / step) * step), TOP), v)


def _values():
    """Pairs of bf16 values whose sums are the pre-activations."""
    pairs = [(0.0, 0.0)]
    for e in range(-44, 37):
        for a in (1.0, 1.3125, 1.9921875):
            pairs += [(a * 2.0 ** e, s * 2.0 ** (e - k)) for k in (8, 9, 10, 11) for s in (1.0, -1.0, 1.5)]
    top = 2.0 ** 33 - 2.0 ** 25
    pairs += [(top, b * 2.0 ** 20) for b in (0, 8, 12, 15, 16, 17, 20, 23, 24, 25, 28, 31, 32, 33)]
    pairs += [(1.5 * 2.0 ** 127, 0.0), (2.0 ** 100, 2.0 ** 99)]
    return [(s * a, s * b) for a, b in pairs for s in (1.0, -1.0)]


def _run(pairs, T):
    """Saved g and u and dx of rows that hold a pair each, T rows a call."""
    eye = torch.eye(D, dtype=torch.bfloat16, device="cuda")
    both = eye.clone()
    both[0, 1] = 1  # pre-activation 0 is x0 + x1
    st = B.new_status()
    got = []
    for i in range(0, len(pairs), T):
        x = torch.zeros(T, D, dtype=torch.bfloat16)
        some = torch.tensor(pairs[i:i + T], dtype=torch.float64)
        x[:len(some), :2] = some.to(torch.bfloat16)
        assert torch.allclose(x[:len(some), :2].double(), some, rtol=0, atol=0, equal_nan=True)  # bf16 holds them
        x = x.cuda()
        dy = torch.zeros_like(x)
        dy[:, 0] = 1
        _, saved = B.olive_gated_mlp_fwd(x, both, both, eye, save=True, dev_status=st)
        dx = B.olive_gated_mlp_bwd(dy, x, both, both, eye, saved, need_dW=False, dev_status=st)[0]
        got.append((saved[0, :len(some), 0], saved[1, :len(some), 0], dx[:len(some), 0]))
    assert B.status_bits(st) == []
    return [torch.cat(t) for t in zip(*got)]


# few rows (one kernel, value by value) and many (another, two values at once)
@pytest.mark.parametrize("T", [16, 64, 300])
def test_what_is_saved(T):
    pairs = _values()
    g, u, dx = _run(pairs, T)
    want = torch.tensor([_held(a + b) for a, b in pairs], dtype=torch.float64)
    assert torch.equal(_decode(g), want) and torch.equal(g, u)
    s = torch.sigmoid(want)
    terms = torch.stack((want * (s + want * s * (1 - s)), want * s))  # dg = u act'(g), du = act(g)
    ref = terms.sum(0)
    assert ((dx.cpu().double() - ref).abs() <= 2.1 * 2.0 ** -8 * terms.abs().sum(0) + 1e-38).all()


@pytest.mark.parametrize("T", [16, 300])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_what_is_not_finite(T, bad):
    g, u, dx = _run([(1.0, 0.0), (bad, 0.0), (2.0, 0.0)], T)
    got = _decode(g)
    assert torch.isnan(got).tolist() == [False, True, False] and torch.equal(g, u)
    assert torch.isnan(dx).tolist() == [False, True, False]
