"""Embedding rows and their gradient against the definition in 64 bits.

Tolerances.  A looked-up value is one fp32 product and one rounding.  A gradient's sum runs over at
most 128 tokens in fp32 (then in fp64): 128 2^-24 = 2^-17 of the sum of its terms' magnitudes, and
the rounding to the type, half a last place (eps / 2).
"""

import pytest
import torch

from paper_2609_36246_gb300 import binding as B

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def _case(T, V, d, dtype, ids="skewed", seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    W = torch.randn(V, d, generator=gen, device="cuda").to(dtype)
    dy = torch.randn(T, d, generator=gen, device="cuda").to(dtype)
    u = torch.rand(T, generator=gen, device="cuda", dtype=torch.float64)
    at = {"skewed": ((V + 1) ** u - 1).long(), "even": (u * V).long(), "one": torch.full_like(u, V // 2).long(),
          "last": torch.full_like(u, V - 1).long(), "ends": torch.where(u < 0.5, 0, V - 1)}[ids]
    return W, at.clamp(0, V - 1).to(torch.int32), dy


def _check(W, ids, dy, scale=1.5, grad_dtype=None, n_ids=None, base=None):
    st = B.new_status()
    V, n = W.shape[0], ids.numel() if n_ids is None else min(max(int(n_ids), 0), ids.numel())
    y = B.olive_embedding_fwd(W, ids, scale, n_ids, dev_status=st)
    want = W.double()[ids[:n].long()] * scale
    assert y.dtype == W.dtype and y.shape == (ids.numel(), W.shape[1])
    eps = torch.finfo(W.dtype).eps / 2
    assert ((y[:n].double() - want).abs() <= 1.01 * eps * want.abs()).all() and not y[n:].any()

    grad_dtype = grad_dtype or W.dtype
    out = None if base is None else base.clone()
    more = dict(n_ids=n_ids, grad_dtype=grad_dtype, dev_status=st)
    dW = B.olive_embedding_bwd(dy, ids, V, scale, out=out, accumulate=base is not None, **more)
    want = torch.zeros(W.shape, dtype=torch.float64, device="cuda")
    size = want.clone()
    want.index_add_(0, ids[:n].long(), dy[:n].double() * scale)
    size.index_add_(0, ids[:n].long(), dy[:n].double().abs() * scale)
    if base is not None:
        want, size = want + base.double(), size + base.double().abs()
    eps = torch.finfo(grad_dtype).eps / 2
    assert dW.dtype == grad_dtype
    assert ((dW.double() - want).abs() <= 2.0 ** -17 * size + 1.01 * eps * want.abs()).all()
    again = B.olive_embedding_bwd(dy, ids, V, scale, out=None if base is None else base.clone(),
                                  accumulate=base is not None, **more)
    assert torch.equal(again, dW)
    assert B.status_bits(st) == []
    if base is not None:  # rows that no token names are left
        left = torch.ones(V, dtype=torch.bool, device="cuda")
        left[ids[:n].long()] = False
        assert torch.equal(dW[left], base[left])
    return y, dW


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 64, 1000, 2048, 2049, 5003])
def test_tokens(T, dtype):
    _check(*_case(T, 997, 72, dtype))


@pytest.mark.parametrize("ids", ["skewed", "even", "one", "last", "ends"])
@pytest.mark.parametrize("V", [1, 2, 31, 32, 33, 511, 512, 513, 2**18 - 1, 2**18 + 3])
def test_vocabularies(V, ids):
    _check(*_case(700, V, 24, BF16, ids))


@pytest.mark.parametrize("d", [8, 264, 1016, 1024, 1032, 4096])
@pytest.mark.parametrize("dtype,grad", [(BF16, BF16), (BF16, F32), (F32, BF16), (F32, F32)])
def test_widths_and_types(d, dtype, grad):
    _check(*_case(300, 130, d, dtype), grad_dtype=grad)


@pytest.mark.parametrize("ids", ["skewed", "one", "ends"])
@pytest.mark.parametrize("T", [65536, 65537, 70001])
def test_many_tokens(T, ids):
    _check(*_case(T, 5000, 16, BF16, ids), grad_dtype=F32)


@pytest.mark.parametrize("n", [-3, 0, 1, 777, 1000, 5000])
def test_rows_behind_the_last_token(n):
    """Ids and gradients behind it are not looked at."""
    W, ids, dy = _case(1000, 300, 40, BF16)
    n = max(-3, n)
    ids[min(max(n, 0), 1000):] = -7
    dy[min(max(n, 0), 1000):] = float("nan")
    _check(W, ids, dy, n_ids=torch.tensor([n], dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("grad", [BF16, F32])
@pytest.mark.parametrize("ids", ["skewed", "one"])
def test_added_to_a_gradient(ids, grad):
    W, at, dy = _case(900, 400, 136, BF16, ids)
    _check(W, at, dy, grad_dtype=grad, base=torch.randn(W.shape, device="cuda").to(grad))


def test_ids_outside_the_vocabulary():
    W, ids, dy = _case(200, 50, 64, BF16)
    good = ids.clone()
    ids[[3, 70, 199]] = torch.tensor([-1, 50, 2**31 - 1], dtype=torch.int32, device="cuda")
    st = B.new_status()
    y = B.olive_embedding_fwd(W, ids, dev_status=st)
    assert B.status_bits(st) == ["OLIVE_ERR_TOKEN_RANGE"]
    keep = torch.ones(200, dtype=torch.bool, device="cuda")
    keep[[3, 70, 199]] = False
    assert torch.isnan(y[~keep]).all() and torch.equal(y[keep], B.olive_embedding_fwd(W, good)[keep])
    st = B.new_status()
    dW = B.olive_embedding_bwd(dy, ids, 50, dev_status=st)
    assert B.status_bits(st) == ["OLIVE_ERR_TOKEN_RANGE"]
    want = torch.zeros(50, 64, dtype=torch.float64, device="cuda").index_add_(0, good[keep].long(), dy[keep].double())
    assert ((dW.double() - want).abs() <= 2.0 ** -8 * 1.01 * want.abs() + 1e-3).all()
    assert torch.equal(B.olive_embedding_bwd(dy, ids, 50), dW)  # without a status word


def test_values_that_are_not_finite_stay_in_their_row():
    W, ids, dy = _case(400, 90, 64, BF16, "even")
    clean = B.olive_embedding_bwd(dy, ids, 90)
    dy[17, 3], dy[200, 9] = float("nan"), float("inf")
    dW = B.olive_embedding_bwd(dy, ids, 90)
    bad = torch.zeros(90, 64, dtype=torch.bool, device="cuda")
    bad[ids[17], 3] = bad[ids[200], 9] = True
    assert torch.equal(~torch.isfinite(dW), bad) and torch.equal(dW[~bad], clean[~bad])


def test_no_tokens():
    W, ids, dy = _case(1, 50, 64, BF16)
    assert B.olive_embedding_fwd(W, ids[:0]).shape == (0, 64)
    assert not B.olive_embedding_bwd(dy[:0], ids[:0], 50).any()
    kept = torch.ones(50, 64, dtype=BF16, device="cuda")
    B.olive_embedding_bwd(dy[:0], ids[:0], 50, out=kept, accumulate=True)
    assert bool((kept == 1).all())


def test_autograd_form():
    W, ids, dy = _case(500, 120, 64, BF16)
    W.requires_grad_()
    y = B.embedding(W, ids, 2.0)
    (torch.cat([y, y], 1)[:, 32:96].float() * dy.float()).sum().backward()  # (a view's gradient)
    rolled = torch.cat([dy[:, 32:], dy[:, :32]], 1).contiguous()
    assert torch.equal(W.grad, B.olive_embedding_bwd(rolled, ids, 120, 2.0))
    g, = torch.autograd.grad(B.embedding(W, ids).square().sum(), W, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g.sum(), W)


def test_captured_and_on_another_stream():
    W, ids, dy = _case(3000, 2000, 72, BF16)
    run = lambda: (B.olive_embedding_fwd(W, ids), B.olive_embedding_bwd(dy, ids, 2000))
    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for seed in (4, 5):
        for t, v in zip((W, ids, dy), _case(3000, 2000, 72, BF16, "even", seed)):
            t.copy_(v)
        want = run()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
