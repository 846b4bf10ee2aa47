"""Which norm a call takes where it names none (no GPU needed): the direct calls the centred one, forward
and backward alike, the autograd form the one without centring, forward and backward alike."""

import pytest
import torch

from paper_2609_36246_gb300 import binding as B
from tests import host_calls

BF16 = torch.bfloat16
LAYER, RMS = 0, 1


@pytest.fixture
def rec(monkeypatch):
    return host_calls.recorded(monkeypatch)


def _kinds(rec):
    return [args[7] for name in ("olive_row_norm_fwd", "olive_row_norm_bwd") for args in rec.named(name)]


def test_direct_calls(rec):
    x, w = torch.zeros(5, 64, dtype=BF16), torch.ones(64, dtype=BF16)
    _, h, stats = B.olive_row_norm_fwd(x, w, save=True)
    B.olive_row_norm_bwd(x, h, w, stats)
    assert _kinds(rec) == [LAYER, LAYER]


@pytest.mark.parametrize("given,kind", [({}, RMS), (dict(kind="rms"), RMS), (dict(kind="layer"), LAYER)], ids=str)
def test_autograd_form(rec, given, kind):
    x, w = torch.zeros(5, 64, dtype=BF16, requires_grad=True), torch.ones(64, dtype=BF16)
    B.row_norm(x, w, **given).sum().backward()
    with torch.no_grad():
        B.row_norm(x, w, **given)
    assert _kinds(rec) == [kind, kind, kind]


def test_a_norm_of_no_name_is_refused(rec):
    x, w = torch.zeros(5, 64, dtype=BF16), torch.ones(64, dtype=BF16)
    for call in (B.olive_row_norm_fwd, B.row_norm):
        with pytest.raises((KeyError, ValueError)):
            call(x, w, kind="batch")
    assert not rec.calls
