"""Host-side refusals of the embedding and the rows' norm (no GPU needed): bad pointers, shapes,
alignment, enums and workspaces are rejected with their status before anything is launched, and what
the binding refuses by itself."""

import ctypes

import pytest
import torch

from paper_2609_36246_gb300 import binding as B
from paper_2609_36246_gb300 import build
from tests import host_calls

P = ctypes.c_void_p
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def L():
    build.build()
    return B.lib()


@pytest.fixture(scope="module")
def p():
    # a host buffer used only for its address: validation never dereferences it
    buf = ctypes.create_string_buffer((1 << 16) + 256)
    yield (ctypes.addressof(buf) + 255) // 256 * 256
    del buf


def _launches(status):
    """What a call that passes its checks says where there is no usable device."""
    if torch.cuda.is_available():
        pytest.skip("the addresses here are not the GPU's")
    return status in (7, 8)


def test_workspaces(L):
    size = L.olive_workspace_size
    assert size(14, 1, 4096, 0, 1, 0, 0) > 0 and size(14, 1, 60, 0, 1, 0, 0) == 0 and size(14, 1, 16392, 0, 1, 0, 0) == 0
    assert size(15, 100, 64, 0, 500, 0, 0) > 0 and size(15, 0, 64, 0, 500, 0, 0) == 0
    assert size(15, 100, 60, 0, 500, 0, 0) == 0 and size(15, 100, 64, 0, 0, 0, 0) == 0
    assert size(15, 10000, 64, 0, 500, 0, 0) > size(15, 100, 64, 0, 500, 0, 0)
    assert all(size(op, 100, 64, 0, 500, 0, 0) % 256 == 0 for op in (14, 15))


def test_embedding(L, p):
    def fwd(**kw):
        a = dict(W=p, ids=p, n=None, T=5, V=50, d=64, scale=1.0, out=p, dt=0)
        a.update(kw)
        return L.olive_embedding_fwd(P(a["W"]), P(a["ids"]), P(a["n"]), a["T"], a["V"], a["d"], a["scale"], P(a["out"]),
                                     a["dt"], None, None)

    assert all(fwd(**{k: None}) == 1 for k in ("W", "ids", "out"))
    assert fwd(dt=2) == 1 and fwd(scale=float("nan")) == 1 and fwd(scale=float("inf")) == 1
    assert fwd(T=-1) == 2 and fwd(V=0) == 2 and fwd(d=0) == 2 and fwd(d=1 << 21) == 2
    assert fwd(T=2**31 - 1, d=1 << 20) == 2  # more blocks than a grid has
    assert fwd(d=60) == 3 and fwd(W=p + 8) == 3 and fwd(out=p + 4) == 3
    assert _launches(fwd()) and _launches(fwd(n=p, dt=1)) and _launches(fwd(T=0, ids=None, out=None))

    ws = L.olive_workspace_size(15, 5, 64, 0, 50, 0, 0)

    def bwd(**kw):
        a = dict(dy=p, ids=p, n=None, T=5, V=50, d=64, scale=1.0, dW=p, dt=0, gt=1, acc=0, ws=p, size=ws)
        a.update(kw)
        return L.olive_embedding_bwd(P(a["dy"]), P(a["ids"]), P(a["n"]), a["T"], a["V"], a["d"], a["scale"], P(a["dW"]),
                                     a["dt"], a["gt"], a["acc"], P(a["ws"]), a["size"], None, None)

    assert all(bwd(**{k: None}) == 1 for k in ("dy", "ids", "dW"))
    assert bwd(dt=2) == 1 and bwd(gt=-1) == 1 and bwd(acc=2) == 1 and bwd(scale=float("nan")) == 1
    assert bwd(T=-1) == 2 and bwd(V=0) == 2 and bwd(d=0) == 2 and bwd(T=2**31 - 1, d=1 << 20) == 2
    assert bwd(d=60) == 3 and bwd(dy=p + 8) == 3 and bwd(dW=p + 8) == 3
    assert bwd(size=ws - 256) == 9 and bwd(ws=None) == 9 and bwd(ws=p + 16) == 9
    assert _launches(bwd()) and _launches(bwd(acc=1)) and _launches(bwd(T=0, dy=None, ids=None, ws=None, acc=1))


def test_row_norm(L, p):
    q = p + 4096

    def fwd(**kw):
        a = dict(x=p, res=None, w=p, b=None, T=5, d=64, eps=1e-6, kind=0, y=p, sum=None, stats=None, dt=0)
        a.update(kw)
        return L.olive_row_norm_fwd(P(a["x"]), P(a["res"]), P(a["w"]), P(a["b"]), a["T"], a["d"], a["eps"], a["kind"],
                                    P(a["y"]), P(a["sum"]), P(a["stats"]), a["dt"], None)

    assert all(fwd(**{k: None}) == 1 for k in ("x", "w", "y"))
    assert fwd(dt=2) == 1 and fwd(kind=2) == 1 and fwd(eps=-1.0) == 1 and fwd(eps=float("nan")) == 1
    assert fwd(res=p) == 1 and fwd(sum=q) == 1 and fwd(res=p, sum=p) == 1  # (y and the sum in one place)
    assert fwd(T=-1) == 2 and fwd(d=0) == 2 and fwd(d=16392) == 2
    assert fwd(d=60) == 3 and all(fwd(**{k: p + 8}) == 3 for k in ("x", "w", "b", "y"))
    assert fwd(res=p + 8, sum=q) == 3 and fwd(res=p, sum=q + 8) == 3
    assert _launches(fwd()) and _launches(fwd(res=p, sum=q, b=p, stats=p, kind=1)) and _launches(fwd(T=0, x=None, y=None))

    ws = L.olive_workspace_size(14, 1, 64, 0, 1, 0, 0)

    def bwd(**kw):
        a = dict(dy=p, h=p, w=p, stats=p, gs=None, T=5, d=64, kind=1, dx=p, dw=p, db=None, dt=0, ws=p, size=ws)
        a.update(kw)
        return L.olive_row_norm_bwd(P(a["dy"]), P(a["h"]), P(a["w"]), P(a["stats"]), P(a["gs"]), a["T"], a["d"],
                                    a["kind"], P(a["dx"]), P(a["dw"]), P(a["db"]), a["dt"], P(a["ws"]), a["size"], None)

    assert all(bwd(**{k: None}) == 1 for k in ("dy", "h", "w", "stats", "dx", "dw"))
    assert bwd(dt=2) == 1 and bwd(kind=-1) == 1
    assert bwd(T=-1) == 2 and bwd(d=16392) == 2
    assert bwd(d=60) == 3 and all(bwd(**{k: p + 8}) == 3 for k in ("dy", "h", "w", "gs", "dx"))
    assert bwd(size=ws - 256) == 9 and bwd(ws=None) == 9
    assert _launches(bwd()) and _launches(bwd(gs=p, db=p)) and _launches(bwd(T=0, dy=None, h=None, stats=None, dx=None))


# ------------------------------------------------------- the Python calls ---

@pytest.fixture
def rec(monkeypatch):
    return host_calls.recorded(monkeypatch)


def _calls():
    """Each call as (its tensors, the call of them)."""
    r = lambda *s: torch.randn(*s).to(BF16)
    ids = lambda n: torch.zeros(n, dtype=torch.int32)
    extra = lambda: dict(ws=torch.zeros(4096, dtype=torch.uint8), st=ids(1))
    e = extra()
    yield dict(W=r(50, 64), ids=ids(5), n=ids(1), out=r(5, 64), st=e["st"]), lambda t: \
        B.olive_embedding_fwd(t["W"], t["ids"], n_ids=t["n"], out=t["out"], dev_status=t["st"])
    yield dict(dy=r(5, 64), ids=ids(5), n=ids(1), out=r(50, 64), **extra()), lambda t: \
        B.olive_embedding_bwd(t["dy"], t["ids"], 50, n_ids=t["n"], out=t["out"], ws=t["ws"], dev_status=t["st"])
    yield dict(x=r(5, 64), w=r(64), b=r(64), res=r(5, 64), y=r(5, 64), s=r(5, 64)), lambda t: \
        B.olive_row_norm_fwd(t["x"], t["w"], t["b"], t["res"], out=t["y"], sum_out=t["s"])
    yield dict(dy=r(5, 64), h=r(5, 64), w=r(64), stats=torch.zeros(2, 5), g=r(5, 64), dx=r(5, 64), ws=e["ws"]), lambda t: \
        B.olive_row_norm_bwd(t["dy"], t["h"], t["w"], t["stats"], t["g"], out=t["dx"], ws=t["ws"])


def test_tensors_of_another_device_or_layout_are_refused(rec):
    for tensors, call in _calls():
        call(tensors)
        made = len(rec.calls)
        for name, t in tensors.items():
            rec.place(t, 1)
            with pytest.raises(TypeError):
                call(tensors)
            rec.place(t, 0)
            if t.dim() == 2:
                with pytest.raises((TypeError, ValueError)):
                    call({**tensors, name: t.t().contiguous().t()})
        assert len(rec.calls) == made


def test_shapes_and_types_are_refused(rec):
    for tensors, call in _calls():
        call(tensors)
        made = len(rec.calls)
        for name, t in tensors.items():
            if name in ("ws", "st"):
                continue
            with pytest.raises(TypeError):
                call({**tensors, name: t.to(torch.float16)})
            if name != "W":  # (a vocabulary may have any size)
                with pytest.raises(ValueError):
                    call({**tensors, name: torch.cat([t, t])})
        assert len(rec.calls) == made
    dy, ids = torch.zeros(5, 64), torch.zeros(5, dtype=torch.int32)
    for bad in (lambda: B.olive_embedding_bwd(dy, ids, 50, accumulate=True),
                lambda: B.olive_row_norm_fwd(dy, torch.zeros(64), sum_out=dy)):
        with pytest.raises(ValueError):
            bad()


def test_gradients_off_the_16_byte_rule_are_copied(rec):
    W = torch.zeros(50, 64, dtype=BF16, requires_grad=True)
    y = B.embedding(W, torch.zeros(5, dtype=torch.int32))
    y.backward(torch.ones(5 * 64 + 1, dtype=BF16)[1:].view(5, 64))
    x = torch.zeros(5, 64, dtype=BF16, requires_grad=True)
    B.row_norm(x, torch.ones(64, dtype=BF16)).backward(torch.ones(64, 5, dtype=BF16).t())
    for name in ("olive_embedding_bwd", "olive_row_norm_bwd"):
        (args,) = rec.named(name)
        assert args[0] % 16 == 0
