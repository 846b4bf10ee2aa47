"""Host-side refusals of the calls around the loss (no GPU needed): bad pointers, shapes, alignment,
enums and workspaces are rejected with their status before anything is launched."""

import ctypes

import pytest
import torch

from paper_2609_36246_gb300 import binding as B
from paper_2609_36246_gb300 import build

P = ctypes.c_void_p


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
    assert size(10, 100, 64, 0, 72, 0, 0) >= 2 * 100 * 72
    assert size(11, 100, 64, 0, 72, 1, 0) >= 3 * 2 * 100 * 72
    assert size(10, 0, 64, 0, 72, 0, 0) == 0 and size(10, 1, 60, 0, 72, 0, 0) == 0 and size(10, 1, 64, 0, 70, 0, 0) == 0
    assert size(12, 1, 128, 0, 1, 0, 0) > 0 and size(12, 1, 264, 0, 1, 0, 0) == 0 and size(12, 1, 12, 0, 1, 0, 0) == 0
    assert size(13, 1, 0, 0, 1, 0, 0) > 0 and size(13, 0, 0, 0, 1, 0, 0) == 0
    assert size(13, 2000, 0, 0, 1, 0, 0) > size(13, 100, 0, 0, 1, 0, 0)
    assert all(size(op, 100, 64, 0, 72, 1, 0) % 256 == 0 for op in (10, 11, 12, 13))


def test_gated_mlp(L, p):
    ws = L.olive_workspace_size(11, 100, 64, 0, 72, 1, 0)

    def fwd(**kw):
        a = dict(x=p, wg=p, wu=p, wd=p, r=None, T=100, d=64, f=72, act=0, y=p, saved=p, ws=p, n=ws)
        a.update(kw)
        return L.olive_gated_mlp_fwd(*[P(a[k]) for k in ("x", "wg", "wu", "wd", "r")], a["T"], a["d"], a["f"],
                                     a["act"], P(a["y"]), P(a["saved"]), P(a["ws"]), a["n"], None, None)

    assert all(fwd(**{k: None}) == 1 for k in ("x", "wg", "wu", "wd", "y"))
    assert fwd(act=2) == 1 and fwd(act=-1) == 1
    assert fwd(T=-1) == 2 and fwd(d=0) == 2 and fwd(f=0) == 2 and fwd(d=1 << 21) == 2
    assert fwd(d=60) == 3 and fwd(f=68) == 3
    assert all(fwd(**{k: p + 8}) == 3 for k in ("x", "wg", "wu", "wd", "r", "y", "saved"))
    assert fwd(n=64) == 9 and fwd(ws=p + 16) == 9 and fwd(ws=None) == 9
    assert _launches(fwd()) and _launches(fwd(saved=None)) and _launches(fwd(T=0, x=None, y=None, ws=None))


def test_gated_mlp_backward(L, p):
    ws = L.olive_workspace_size(11, 100, 64, 0, 72, 1, 0)

    def bwd(**kw):
        a = dict(dy=p, x=p, wg=p, wu=p, wd=p, saved=p, T=100, d=64, f=72, act=0, dx=p, dg=p, du=p, dd=p, dt=0, ws=p, n=ws)
        a.update(kw)
        return L.olive_gated_mlp_bwd(*[P(a[k]) for k in ("dy", "x", "wg", "wu", "wd", "saved")], a["T"], a["d"],
                                     a["f"], a["act"], *[P(a[k]) for k in ("dx", "dg", "du", "dd")], a["dt"],
                                     P(a["ws"]), a["n"], None, None)

    assert all(bwd(**{k: None}) == 1 for k in ("dy", "x", "wg", "wu", "wd", "saved", "dg", "du", "dd"))
    assert bwd(dx=None, dg=None, du=None, dd=None) == 1 and bwd(dt=2) == 1 and bwd(act=5) == 1
    assert bwd(T=-1) == 2 and bwd(d=0) == 2
    assert bwd(d=60) == 3 and bwd(f=68) == 3
    assert all(bwd(**{k: p + 4}) == 3 for k in ("dy", "x", "wg", "wu", "wd", "saved", "dx", "dg", "du", "dd"))
    assert bwd(n=ws - 256) == 9
    assert _launches(bwd()) and _launches(bwd(dx=None)) and _launches(bwd(dg=None, du=None, dd=None))


def test_qk_norm_rope(L, p):
    def call(bwd=False, **kw):
        a = dict(q=p, k=p, wq=p, wk=p, cos=p, sin=p, pos=p, yq=p, yk=p, gq=p, gk=p, dwq=p, dwk=p, ts=256, hs=64,
                 Hq=3, Hk=1, eps=1e-6, P=9, T=5, D=64, R=64, inter=0, dt=0, ws=p, n=1 << 22)
        a.update(kw)
        view = lambda k: (P(a[k]), a["ts"], a["hs"])
        mid = (a["Hq"], a["Hk"], P(a["wq"]), P(a["wk"]), a["eps"], P(a["cos"]), P(a["sin"]), P(a["pos"]), a["P"], a["T"],
               a["D"], a["R"], a["inter"])
        if bwd:
            return L.olive_qk_norm_rope_bwd(*view("gq"), *view("gk"), *view("q"), *view("k"), *mid, *view("yq"),
                                            *view("yk"), P(a["dwq"]), P(a["dwk"]), a["dt"], P(a["ws"]), a["n"], None, None)
        return L.olive_qk_norm_rope_fwd(*view("q"), *view("k"), *mid, *view("yq"), *view("yk"), a["dt"], None, None)

    for b in (False, True):
        assert all(call(b, **{k: None}) == 1 for k in ("q", "k", "wq", "wk", "cos", "sin", "pos", "yq", "yk"))
        assert call(b, dt=2) == 1 and call(b, inter=2) == 1
        assert call(b, eps=-1e-6) == 1 and call(b, eps=float("nan")) == 1 and call(b, eps=float("inf")) == 1
        assert call(b, T=-1) == 2 and call(b, D=264) == 2 and call(b, R=72) == 2 and call(b, R=-8) == 2
        assert call(b, P=0) == 2 and call(b, Hq=0, Hk=0) == 2 and call(b, Hq=-1) == 2 and call(b, ts=-256) == 2
        assert call(b, D=60, R=0) == 3 and call(b, R=20) == 3 and call(b, ts=260) == 3 and call(b, hs=68) == 3
        assert all(call(b, **{k: p + 8}) == 3 for k in ("q", "k", "wq", "wk", "cos", "sin", "yq", "yk"))
        assert _launches(call(b)) and _launches(call(b, Hk=0, k=None, wk=None, yk=None, gk=None))
        assert _launches(call(b, R=0, cos=None, sin=None))
        assert _launches(call(b, T=0, q=None, k=None, yq=None, yk=None, gq=None, gk=None, pos=None))
    assert call(True, gq=None) == 1 and call(True, dwq=None) == 1 and call(True, dwk=None) == 1
    assert call(True, gk=p + 8) == 3 and call(True, n=64) == 9 and call(True, ws=None) == 9


def test_packed_positions(L, p):
    assert L.olive_packed_positions(None, 1, 1, P(p), None) == 1 and L.olive_packed_positions(P(p), 1, 1, None, None) == 1
    assert L.olive_packed_positions(P(p), 0, 1, P(p), None) == 2 and L.olive_packed_positions(P(p), 1, 0, P(p), None) == 2
    assert _launches(L.olive_packed_positions(P(p), 1, 1, P(p), None))


def test_grad_clip(L, p):
    ws = L.olive_workspace_size(13, 2, 0, 0, 1, 0, 0)

    def call(src=(p, p + 4096), dst=(p, p + 4096), num=(10, 20), dt=(0, 1), n=2, limit=1.0, norm=p, size=ws):
        arr = lambda t, v: (t * 2)(*v) if v is not None else None
        return L.olive_grad_clip(arr(P, src), arr(P, dst), arr(ctypes.c_int64, num), arr(ctypes.c_int32, dt), n, limit,
                                 P(norm), P(p), size, None)

    assert call(n=-1) == 2 and call(num=(10, -1)) == 2
    assert call(src=None) == 1 and call(num=None) == 1 and call(dt=None) == 1 and call(norm=None) == 1
    assert call(dt=(0, 2)) == 1 and call(src=(p, None)) == 1 and call(dst=(None, p)) == 1
    assert call(limit=0.0) == 1 and call(limit=-1.0) == 1 and call(limit=float("nan")) == 1
    assert call(src=(p + 1, p)) == 3 and call(src=(p, p + 2)) == 3 and call(dst=(p, p + 2)) == 3
    assert call(size=64) == 9
    assert _launches(call()) and _launches(call(src=(p + 2, p + 4), dst=(p + 2, p + 4)))
    assert _launches(call(src=(None, p), dst=(None, p), num=(0, 5))) and _launches(call(dst=None))
