"""Attention with caps of every size against the definition in 64 bits.

Tolerances.  A capped score is off by a part of itself, whatever the cap: z / cap, the tanh and its
product with the cap are some ten roundings of 2^-24 and special functions within 2^-22, below 2^-20 of
the score together.  Scores of large caps have the tolerances of scores without one, whose 2^-16 of
A = scale sum |q||k| >= |z| is a sum of 128 terms' 2^-17 and has room for 2^-20 |z|: such a cap changes
z by less than 1e-4 of it here.  Scores of small caps have those of the capped score.
"""

import pytest

from tests import test_packed_attention_gpu as base

pytestmark = pytest.mark.gpu


def _compare(s, tolerances):
    ref = base._reference(s, True)
    ref.update({n: t for n, t in tolerances.items() if n.startswith("tol_")})
    o, lse = base._forward(s)
    base._near(o, ref, "o")
    base._near(lse, ref, "lse")
    for name, g in zip(("dq", "dk", "dv"), base._backward(s, o, lse)):
        base._near(g, ref, name)


@pytest.mark.parametrize("cap", [1e4, 1e6, 1e9, 1e25, 3.4e38])
@pytest.mark.parametrize("lens", [[20], [100], [300], [12, 1, 640, 0, 130]], ids=str)
@pytest.mark.parametrize("hq,hk,D", [(4, 2, 128), (3, 3, 40)])
def test_large(lens, hq, hk, D, cap):
    """A cap far above the scores, a way to say that there is none, changes them by less than their rounding."""
    s = base._case(lens, hq, hk, D, pad=5, sharp=2.0, cap=cap)
    plain = {**s, "more": {**s["more"], "cap": 0.0}}
    _compare(s, base._reference(plain, True))


@pytest.mark.parametrize("form", [dict(prefix=140), dict(bias=True), dict(causal=False)], ids=str)
def test_large_in_other_forms(form):
    s = base._case([300, 17, 129], 4, 2, 64, sharp=2.0, cap=1e7, **form)
    plain = {**s, "more": {**s["more"], "cap": 0.0}}
    _compare(s, base._reference(plain, True))


@pytest.mark.parametrize("cap", [1e-42, 1e-30, 0.01, 0.5])
@pytest.mark.parametrize("lens", [[20], [300, 129]], ids=str)
def test_small(lens, cap):
    """Scores that are all at their cap, some that are exactly 0 among them."""
    s = base._case(lens, 4, 2, 64, cap=cap)
    s["q"][3::7, 1] = 0
    _compare(s, {})


@pytest.mark.parametrize("cap", [30.0, 64.0, 65.0, 200.0])
def test_scores_of_every_size_in_a_tile(cap):
    """Rows whose scores are at the cap beside rows whose scores are far below it."""
    s = base._case([300, 90], 4, 2, 128, cap=cap)
    s["q"][1::2] *= 64
    s["q"][2::4] *= 2.0 ** -10
    _compare(s, {})


@pytest.mark.parametrize("form", [dict(cap=100.0), dict(cap=65.0, bias=True, prefix=20), dict(cap=1e5, causal=False)], ids=str)
def test_what_is_not_finite_with_a_wide_cap(form):
    """As with a small one: a bad token behind a sequence's end, or in another one, does not show in a bit."""
    base.test_what_is_not_finite({**form, "sharp": 4.0})


@pytest.mark.parametrize("form", [dict(cap=100.0), dict(cap=70.0, bias=True), dict(prefix=900, cap=100.0)], ids=str)
def test_the_same_bits_whatever_ran_before_with_a_wide_cap(form):
    base.test_the_same_bits_whatever_ran_before({**form, "sharp": 4.0})
