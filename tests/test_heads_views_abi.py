"""Which views of heads the calls write to, on the host: no two heads may share memory there."""

import ctypes
import itertools
import random

import pytest
import torch

from paper_2609_36246_gb300 import binding as B
from paper_2609_36246_gb300 import build

P = ctypes.c_void_p


@pytest.fixture(scope="module")
def status():
    build.build()
    L = B.lib()
    if torch.cuda.is_available():
        pytest.skip("the addresses here are not the GPU's")
    # a host buffer used only for its address: validation never dereferences it
    buf = ctypes.create_string_buffer(1 << 16)
    p = (ctypes.addressof(buf) + 255) // 256 * 256

    def call(bwd, T, heads, D, q_out, k_out=None, q_in=None):
        plain = (heads * D, D)
        view = lambda strides: (P(p), *(strides or plain))
        mid = (heads, heads, P(p), P(p), 1e-6, P(p), P(p), P(p), 4, T, D, 0, 0)
        outs = (*view(q_out), *view(k_out))
        if bwd:
            return L.olive_qk_norm_rope_bwd(*view(q_in), *view(None), *view(q_in), *view(None), *mid, *outs, P(p), P(p), 0,
                                            P(p), 1 << 22, None, None)
        return L.olive_qk_norm_rope_fwd(*view(q_in), *view(None), *mid, *outs, 0, None, None)

    return call


def _share(T, heads, D, ts, hs):
    starts = sorted(t * ts + h * hs for t, h in itertools.product(range(T), range(heads)))
    return any(b - a < D for a, b in zip(starts, starts[1:]))


@pytest.mark.parametrize("bwd", [False, True])
def test_outputs_whose_heads_share_memory_are_refused(status, bwd):
    for T, heads, D, strides in ((2, 1, 64, (0, 0)), (1, 2, 64, (0, 0)), (5, 3, 64, (0, 64)), (5, 3, 64, (192, 0)),
                                 (5, 3, 64, (184, 64)), (5, 3, 64, (64, 64)), (5, 3, 64, (64, 312)), (1, 3, 64, (0, 56))):
        assert status(bwd, T, heads, D, strides) == 2 and status(bwd, T, heads, D, None, strides) == 2
    # what is read may be one head (or token) for all, and what has no second head has no stride
    assert status(bwd, 5, 3, 64, None, None, (0, 0)) in (7, 8)
    assert status(bwd, 1, 1, 64, (0, 0), (0, 0)) in (7, 8) and status(bwd, 0, 3, 64, (0, 0), (0, 0)) in (7, 8)
    # token by token, head by head, with gaps, woven into one another
    for strides in ((192, 64), (64, 320), (512, 72), (72, 1000), (8 * 40, 64)):
        assert status(bwd, 5, 3, 64, strides, strides) in (7, 8), strides
    assert status(bwd, 2, 2, 64, (192, 128), (128, 192)) in (7, 8)


def test_drawn_strides_against_all_pairs(status):
    rng = random.Random(0)
    seen = [0, 0]
    for _ in range(20000):
        T, heads, D = rng.randint(1, 6), rng.randint(1, 6), 8 * rng.randint(1, 3)
        ts, hs = 8 * rng.randint(0, 24), 8 * rng.randint(0, 24)
        share = _share(T, heads, D, ts, hs)
        seen[share] += 1
        assert (status(False, T, heads, D, (ts, hs)) == 2) == share, (T, heads, D, ts, hs)
    assert min(seen) > 2000
