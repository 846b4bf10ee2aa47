"""Global gradient norm and clipping against 64 bits.

Tolerances.  Squares are summed in fp32 by 32s (32 roundings of 2^-24 at most) and in fp64 beyond,
and the square root halves a relative error: the norm is off by at most 2^-20 and its own rounding;
1e-6 covers it.  A clipped value adds the factor's and its product's rounding in fp32 (2^-23) and
for bf16 its own, half a last place: 2^-8 (8 significant bits).
"""

import pytest
import torch

from paper_2609_36246_gb300 import binding as B

pytestmark = pytest.mark.gpu

SIZES = [(1,), (7,), (8,), (4096,), (4097,), (8191,), (128, 3), (0,), (1000, 257), (3,), (8192, 8)]


def _grads(sizes, dtypes, scale=1.0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(*s, generator=gen, device="cuda") * scale).to(dtypes[i % len(dtypes)]) for i, s in enumerate(sizes)]


def _norm(grads):
    return float(sum(g.double().square().sum() for g in grads)) ** 0.5 if grads else 0.0


def _check(grads, limit, out):
    norm = _norm(grads)
    f = min(1.0, limit / (norm + 1e-6))
    want = [g.double() * f for g in grads]
    got = B.olive_grad_clip(grads, limit, out=out)
    assert got.dtype == torch.float32 and abs(float(got) - norm) <= 1e-6 * norm + 1e-45
    for g, w in zip(grads if isinstance(out, str) else out, want):
        # (a bf16 value's last place; subnormal results round to a multiple of theirs)
        tol = 2.0 ** -8 * 1.01 if g.dtype == torch.bfloat16 else 2e-6
        assert ((g.double() - w).abs() <= tol * w.abs() + (1e-40 if g.dtype == torch.bfloat16 else 1e-44)).all()


@pytest.mark.parametrize("dtypes", [[torch.bfloat16], [torch.float32], [torch.bfloat16, torch.float32]])
@pytest.mark.parametrize("limit", [0.37, 1e9])
@pytest.mark.parametrize("inplace", [True, False])
def test_lists(dtypes, limit, inplace):
    g = _grads(SIZES, dtypes)
    _check(g, limit, "inplace" if inplace else [torch.full_like(t, 5) for t in g])


@pytest.mark.parametrize("n", [1, 47, 48, 49, 511, 512, 513, 1100])
def test_many_tensors(n):
    g = _grads([(1 + (37 * i) % 700,) for i in range(n)], [torch.bfloat16, torch.float32])
    _check(g, 1.0, "inplace")


def test_larger_than_a_pass():
    g = _grads([(5000, 4099), (1,), (4096, 2048)], [torch.float32, torch.bfloat16])
    _check(g, 2.0, "inplace")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("off", [1, 2, 3, 5, 8])
def test_views_that_start_anywhere(dtype, off):
    flat = _grads([(30011,)], [dtype])[0]
    before = flat.clone()
    g = [flat[off:off + 9001], flat[off + 9001:off + 9001 + 20000]]
    _check(g, 0.5, "inplace")
    end = off + 29001
    assert torch.equal(flat[:off], before[:off]) and torch.equal(flat[end:], before[end:])
    # an aligned source into a shifted place, and the other way round
    for a, b in ((0, off), (off, 0)):
        src, dst = before[a:a + 5003], torch.zeros(6000, dtype=dtype, device="cuda")
        _check([src], 0.5, [dst[b:b + 5003]])
        assert float(dst[:b].abs().sum()) == 0 and float(dst[b + 5003:].abs().sum()) == 0


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-22, 1e-18, 1e18, 1e22, 1e30])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_squares_outside_fp32(scale, dtype):
    _check(_grads([(5000,), (77, 33)], [dtype], scale), 1e-3, "inplace")


# the ends of the types' ranges, and both sides of the sums at which the squares are scaled (1e-28
# and 1e36); the norm of the largest ones stays within
# fp32, and 1 / norm, subnormal there, keeps 21 bits
@pytest.mark.parametrize("value,count", [
    (1e-45, 5000), (9.2e-41, 5000), (1.2e-38, 5000), (1.7e-15, 4097), (1.8e-15, 4097), (2.5e-15, 4097), (1e-14, 1), (1.1e-14, 1),
    (1.7e17, 4097), (1.8e17, 4097), (2.5e17, 4097), (9.9e17, 1), (1.01e18, 1), (3.3e38, 1), (1e37, 900)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ends_of_the_range(value, count, dtype):
    g = [torch.full((count,), value, device="cuda").to(dtype)]
    g[0][::3] *= -1
    _check(g, 1.0, "inplace")


@pytest.mark.parametrize("big,small", [(1e-15, 1e-45), (1e-15, 1e-30), (1e-12, 1e-40), (1.5e38, 1e-45), (1e18, 1e-3), (1e18, 1e17)])
def test_ends_of_the_range_within_a_vector(big, small):
    g = torch.full((4000,), small, device="cuda")
    g[5::1000] = big
    _check([g], 1.0, "inplace")


def test_large_beside_small():
    g = _grads([(9000,), (9000,)], [torch.float32])
    g[0] *= 1e25
    g[1] *= 1e-25
    _check(g, 1.0, "inplace")
    assert float(g[0].norm()) <= 1.0 + 1e-5


def test_zeros_and_nothing():
    g = [torch.zeros(1000, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, 5, device="cuda"), -torch.zeros(100, device="cuda")]
    assert float(B.olive_grad_clip(g, 1.0)) == 0 and all(float(t.abs().sum()) == 0 for t in g)
    assert float(B.olive_grad_clip([], 1.0)) == 0
    assert float(B.olive_grad_clip([g[0][:0]], 1.0)) == 0


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("at", [0, 4099])
def test_not_finite(bad, dtype, at):
    """An infinite norm gives the factor 0, a NaN one NaN, as the formula does."""
    g = _grads([(300,), (4100,)], [dtype])
    g[1][at] = bad
    norm = float(B.olive_grad_clip(g, 1.0))
    if bad != bad:
        assert norm != norm and all(torch.isnan(t).all() for t in g)
    else:
        assert norm == float("inf") and float(g[0].abs().max()) == 0 and torch.isnan(g[1][at])


def test_below_the_limit_nothing_changes():
    g = _grads(SIZES, [torch.bfloat16, torch.float32])
    before = [t.clone() for t in g]
    B.olive_grad_clip(g, 1e6)
    assert all(torch.equal(a, b) for a, b in zip(g, before))
    norm = B.olive_grad_clip(g, 0.1, out=None)
    assert abs(float(norm) - _norm(g)) <= 1e-6 * _norm(g) and all(torch.equal(a, b) for a, b in zip(g, before))


def test_same_bits_streams_and_graphs():
    g = _grads(SIZES * 3, [torch.bfloat16, torch.float32])
    out = [torch.empty_like(t) for t in g]
    first = [B.olive_grad_clip(g, 0.7, out=out)] + [t.clone() for t in out]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = [B.olive_grad_clip(g, 0.7, out=out)] + [t.clone() for t in out]
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = B.olive_grad_clip(g, 0.7, out=out)
    for t in out:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(first, again, [norm] + out):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_parameters():
    p = [torch.nn.Parameter(torch.zeros(50, 20, device="cuda")), torch.nn.Parameter(torch.zeros(9, device="cuda"))]
    p[0].grad = torch.ones(50, 20, device="cuda")
    norm = B.clip_grad_norm_(p, 1.0)
    assert abs(float(norm) - 1000 ** 0.5) < 1e-4 and abs(float(p[0].grad.norm()) - 1.0) < 1e-5 and p[1].grad is None


def test_refusals():
    g = _grads([(40, 30)], [torch.float32])
    with pytest.raises(TypeError):
        B.olive_grad_clip([g[0].half()], 1.0)
    with pytest.raises(TypeError):
        B.olive_grad_clip([g[0].t()], 1.0)
    with pytest.raises(TypeError):
        B.olive_grad_clip([g[0].cpu()], 1.0)
    with pytest.raises(TypeError):
        B.olive_grad_clip(g, 1.0, out=[g[0].bfloat16()])
    with pytest.raises(ValueError):
        B.olive_grad_clip(g, 1.0, out=[])
    for limit in (0.0, -1.0, float("nan")):
        with pytest.raises(B.OliveError) as e:
            B.olive_grad_clip(g, limit)
        assert e.value.status == 1
