"""Attention whose blocks take over items of one another, against the definition in 64 bits: more items
than SMs, of long sequences (a block asks when its last copies are issued) and of short ones (it asks
ahead), heads wider than 64 and narrower, two heads, two tiles and heads apart in a block, dk and dv in
one part and in several.  Tolerances as for the other lengths."""

import os

import pytest
import torch

from tests import test_packed_attention_gpu as base

pytestmark = pytest.mark.gpu

LONG = [3000, 2500]  # 43 key tiles, 23 items a head of two tiles, 44 of one
SHORT = [100, 37] * 30


@pytest.mark.parametrize("form", [dict(), dict(cap=20.0, prefix=700), dict(bias=True), dict(causal=False)], ids=str)
@pytest.mark.parametrize("hq,hk,D", [(32, 8, 128), (15, 15, 96), (16, 8, 64)])
def test_long_sequences(form, hq, hk, D):
    base._check(base._case(LONG, hq, hk, D, pad=40, **form))


@pytest.mark.parametrize("form", [dict(), dict(cap=5.0, bias=True), dict(causal=False, prefix=20)], ids=str)
@pytest.mark.parametrize("hq,hk,D", [(8, 4, 128), (5, 5, 128), (12, 4, 72)])
def test_short_sequences(form, hq, hk, D):
    base._check(base._case(SHORT, hq, hk, D, pad=40, **form))


@pytest.mark.parametrize("lens", [[128], [400, 380], [1300], [2560]], ids=str)
@pytest.mark.parametrize("hq,hk", [(7, 1), (32, 2), (9, 3)])
def test_parts_of_the_query_heads(lens, hq, hk):
    """Numbers of key tiles, from the fewest on, that give dk and dv different parts of the heads."""
    base._check(base._case(lens, hq, hk, 32, prefix=100))


@pytest.mark.parametrize("at", [0, 1, 2])
def test_runs_of_empty_sequences(at):
    """Thousands, before, between and behind sequences that do not begin at a multiple of four."""
    lens = [[5, 130], [17, 1]]
    lens.insert(at, [0] * 5000)
    base._check(base._case(sum(lens, []), 2, 1, 64, pad=7, prefix=3))


def test_empty_sequences_between_tokens_cost_no_more_than_before_them():
    """The same items either way: a token's sequence is not looked for by counting."""
    best = []
    for lens in ([0] * 30000 + [4001, 4000], [4001] + [0] * 30000 + [4000]):
        s = base._case(lens, 4, 4, 64)
        o, lse = base._forward(s)
        base._backward(s, o, lse)
        times = []
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            base._backward(s, o, lse)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        best.append(min(times))
    assert best[1] < 1.5 * best[0]


def _as(limit_ms, run):
    old = os.environ.get("OLIVE_WAIT_LIMIT_MS")
    os.environ["OLIVE_WAIT_LIMIT_MS"] = str(limit_ms)
    try:
        out = run()
        torch.cuda.synchronize()
        return out
    finally:
        del os.environ["OLIVE_WAIT_LIMIT_MS"]
        if old is not None:
            os.environ["OLIVE_WAIT_LIMIT_MS"] = old


@pytest.mark.parametrize("causal", [True, False])
def test_an_item_longer_than_the_limit_of_a_wait(causal):
    """The limit is that of a wait for the next tile, not of an item: a row's 260000 keys take some
    milliseconds, and no wait among them one.  (The last item has one tile of rows, so half of its block
    waits for the other half.)"""
    n = 262144 - 200
    s = base._case([n], 1, 1, 64, causal=causal)

    def run():
        o, lse = base._forward(s)
        return (o, lse, *base._backward(s, o, lse))

    want = _as(1000, run)
    got = _as(1, run)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_limit_that_means_none():
    """2^50 ms are 15625 2^56 ns: times the 256 that an item of 255 tiles has, they must not become 0."""
    s = base._case([255 * 128], 2, 2, 64)

    def run():
        o, lse = base._forward(s)
        return (o, lse, *base._backward(s, o, lse))

    want = _as(1000, run)
    assert all(torch.equal(a, b) for a, b in zip(_as(2 ** 50, run), want))


def test_prefix_ends_outside_the_sequence():
    """Before its beginning: no key is seen by all rows; behind its end: all are.  However far outside."""
    s = base._case([50, 200, 3], 4, 2, 64, prefix=0)
    start, end = s["cu"][:-1], s["cu"][1:]
    for given, as_if in (([-2**31] * 3, start), ([-1, -2**31 + 5, 7], start), ([2**31 - 1] * 3, end)):
        res = []
        for ends in (torch.tensor(given, dtype=torch.int32, device="cuda"), as_if.clone()):
            s["more"]["prefix_end"] = ends
            o, lse = base._forward(s)
            res.append((o, lse, *base._backward(s, o, lse)))
        assert all(torch.equal(a, b) for a, b in zip(*res))
