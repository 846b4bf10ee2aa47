"""The embedding's gradient around the numbers of tokens from which the sort takes larger tiles.

Tolerances.  A unit's up to 128 tokens are added in turn in fp32, the units of a run with a running
compensation: (127 + 2) 2^-24 of the sum of the terms' magnitudes, and terms of 2^-48 a unit, below 2^-16
together; the rounding to the type adds half a last place.
"""

import pytest
import torch

from paper_2609_36246_gb300 import binding as B
from tests import test_embedding_gpu as base

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ids", ["skewed", "even", "one"])
@pytest.mark.parametrize("T", [131072, 131073, 2**20, 2**20 + 1, 2**21 + 77])
def test_tiles_of_the_sort(T, ids):
    W, at, dy = base._case(T, 5000, 16, base.BF16, ids)
    got = B.olive_embedding_bwd(dy, at, 5000, 1.5, grad_dtype=base.F32)
    want = torch.zeros(W.shape, dtype=torch.float64, device="cuda")
    size = want.clone()
    want.index_add_(0, at.long(), dy.double() * 1.5)
    size.index_add_(0, at.long(), dy.double().abs() * 1.5)
    assert bool(((got.double() - want).abs() <= 2.0 ** -16 * size + 2.0 ** -24 * 1.01 * want.abs()).all())
    assert torch.equal(B.olive_embedding_bwd(dy, at, 5000, 1.5, grad_dtype=base.F32), got)
