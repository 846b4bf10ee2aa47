"""Forward-mode differentiation (no GPU needed): the autograd forms have no tangents, so a call with one
is refused, whether autograd is on or off, and never answered without it."""

import contextlib

import pytest
import torch
from torch.autograd import forward_ad

from paper_2609_36246_gb300 import binding as B
from tests import host_calls

BF16, I32 = torch.bfloat16, torch.int32

with forward_ad.dual_level():  # (the first compiles torch functions from their sources, which the recorder replaces)
    forward_ad.make_dual(torch.ones(1), torch.ones(1))


@pytest.fixture
def rec(monkeypatch):
    return host_calls.recorded(monkeypatch)


def _forms():
    """Each form as (its differentiable tensors, the call of them)."""
    r = lambda *s: torch.randn(*s).to(BF16)
    cu = torch.tensor([0, 5], dtype=I32)
    yield dict(x=r(5, 64), w=r(64), b=r(64), res=r(5, 64)), lambda t: B.row_norm(t["x"], t["w"], t["b"], t["res"])
    yield dict(x=r(5, 64), Wg=r(128, 64), Wu=r(128, 64), Wd=r(64, 128), res=r(5, 64)), lambda t: \
        B.gated_mlp(t["x"], t["Wg"], t["Wu"], t["Wd"], t["res"])
    yield dict(W=r(50, 64)), lambda t: B.embedding(t["W"], torch.zeros(5, dtype=I32))
    yield dict(q=r(5, 4, 64), k=r(5, 2, 64), v=r(5, 2, 64)), lambda t: B.packed_attention(t["q"], t["k"], t["v"], cu)


@pytest.mark.parametrize("off", [False, True])
def test_tangents_are_refused(rec, off):
    with torch.no_grad() if off else contextlib.nullcontext():
        for tensors, call in _forms():
            call(tensors)
            with forward_ad.dual_level():
                call(tensors)  # (a level without tangents changes nothing)
                for name, t in tensors.items():
                    dual = forward_ad.make_dual(t, torch.ones_like(t))
                    with pytest.raises((RuntimeError, NotImplementedError)):
                        call({**tensors, name: dual})


def test_nothing_is_kept_where_autograd_is_off(rec):
    with torch.no_grad():
        B.row_norm(torch.zeros(5, 64, dtype=BF16, requires_grad=True), torch.ones(64, dtype=BF16))
    (args,) = rec.named("olive_row_norm_fwd")
    assert args[10] is None  # the rows' statistics
