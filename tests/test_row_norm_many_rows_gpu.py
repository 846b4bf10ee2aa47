"""Weights' gradients of the rows' norm over many rows against the definition in 64 bits.

Tolerances.  A thread adds T / groups rows in turn in fp32, at least 152 groups: at most 1725 rows at
2^18, and some 40 sums of groups: (1725 + 40) 2^-24 < 2^-13 of the sum of the terms' magnitudes.  A term
dy n is within 2^-16 of its own, as for few rows.
"""

import pytest
import torch

from paper_2609_36246_gb300 import binding as B

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
T, EPS = 2 ** 18 + 3, 1e-5


@pytest.mark.parametrize("d,dtype", [(64, F32), (1000, BF16), (2048, F32), (4096, BF16), (8192, BF16)])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_weights_gradients(d, dtype, kind):
    gen = torch.Generator(device="cuda").manual_seed(d)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda", dtype=F32).to(dtype)
    x, w, b = r(T, d), 1 + r(d) / 4, r(d)
    dy = (r(T, d) + 0.5).to(dtype)  # (sums that grow with the rows)
    y, h, stats = B.olive_row_norm_fwd(x, w, b, None, EPS, kind, save=True)
    _, dw, db = B.olive_row_norm_bwd(dy, h, w, stats, None, kind)
    want = [torch.zeros(d, dtype=torch.float64, device="cuda") for _ in range(4)]  # dw, db and their terms' magnitudes
    for i in range(0, T, 1 << 14):
        f, g = x[i:i + (1 << 14)].double(), dy[i:i + (1 << 14)].double()
        m = f.mean(-1, keepdim=True) if kind == "layer" else 0
        n = (f - m) / ((f - m).square().mean(-1, keepdim=True) + EPS).sqrt()
        N = n.abs() + (f.abs().mean(-1, keepdim=True) if kind == "layer" else 0)
        for t, more in zip(want, ((g * n).sum(0), g.sum(0), (g.abs() * N).sum(0), g.abs().sum(0))):
            t += more
    for got, ref, size in ((dw, want[0], want[2]), (db, want[1], want[3])):
        assert bool(((got.double() - ref).abs() <= (2.0 ** -13 + 2.0 ** -16) * size + 2.0 ** -24 * ref.abs()).all())
