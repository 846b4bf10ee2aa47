"""Host-side refusals of the attention inside packed sequences (no GPU needed): bad pointers, shapes,
strides, forms and workspaces are rejected with their status before anything is launched, and what
the binding refuses by itself."""

import ctypes
import math

import pytest
import torch

from paper_2609_36246_gb300 import binding as B
from paper_2609_36246_gb300 import build
from tests import host_calls

P = ctypes.c_void_p
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


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


def test_workspace(L):
    size = lambda T, D=64, Hk=2, Hq=4: L.olive_workspace_size(16, T, D, Hk, Hq, 0, 0)
    assert size(100) >= 8 * 100 * 4 and size(100) % 256 == 0
    assert size(0) == 0 and size(100, D=60) == 0 and size(100, D=136) == 0 and size(100, Hk=0) == 0
    assert size(100, Hk=3) == 0 and size(100, Hq=1) == 0 and size(100, Hq=4098) == 0 and size(2**30 + 1) == 0
    # few key tiles: parts of the query heads' sums as well
    assert size(1000) >= 8 * 1000 * 4 + 8 * 2 * 1000 * 2 * 64 and size(100_000) < 8 * 100_000 * 4 + 4096


def test_calls(L, p):
    q2 = p + 8192
    views = ("do", "q", "k", "v", "o")

    def call(bwd, **kw):
        a = dict(do=p, q=p, k=p, v=p, o=q2, dq=q2, dk=q2, dv=q2, lse=p, ts=512, hs=64, ots=512, ohs=64, Hq=4, Hk=2, cu=p,
                 S=3, T=50, D=64, scale=0.125, causal=1, prefix=None, cap=0.0, slopes=None, ws=p, n=1 << 20)
        a.update(kw)
        view = lambda k: (P(a[k]), a["ts"], a["hs"])
        out = lambda k: (P(a[k]), a["ots"], a["ohs"])
        form = (a["Hq"], a["Hk"], P(a["cu"]), a["S"], a["T"], a["D"], a["scale"], a["causal"], P(a["prefix"]), a["cap"],
                P(a["slopes"]))
        if bwd:
            return L.olive_packed_attention_bwd(*view("do"), *view("q"), *view("k"), *view("v"), *view("o"), P(a["lse"]),
                                                *form, *out("dq"), *out("dk"), *out("dv"), P(a["ws"]), a["n"], None, None)
        return L.olive_packed_attention_fwd(*view("q"), *view("k"), *view("v"), *form, *out("o"), P(a["lse"]), None, None)

    for bwd in (False, True):
        assert all(call(bwd, **{k: None}) == 1 for k in (views if bwd else ("q", "k", "v", "o")) + ("cu",))
        assert call(bwd, causal=2) == 1 and call(bwd, causal=-1) == 1
        assert all(call(bwd, scale=x) == 1 for x in (0.0, -1.0, math.nan, math.inf))
        assert all(call(bwd, cap=x) == 1 for x in (-1.0, math.nan, math.inf))
        assert call(bwd, T=-1) == 2 and call(bwd, T=2**30 + 1) == 2 and call(bwd, S=0) == 2
        assert call(bwd, D=0) == 2 and call(bwd, D=136) == 2
        assert call(bwd, Hk=0) == 2 and call(bwd, Hq=1) == 2 and call(bwd, Hq=5) == 2 and call(bwd, Hq=4098) == 2
        assert call(bwd, T=2**30, S=2**20, Hq=4096, Hk=4096) == 2  # more blocks than a grid has
        assert call(bwd, ts=0) == 2 and call(bwd, ts=-512) == 2 and call(bwd, hs=-64) == 2 and call(bwd, ts=2**39) == 2
        assert call(bwd, ohs=0) == 2 and call(bwd, ots=128) == 2  # an output whose heads share memory
        assert call(bwd, D=60) == 3 and call(bwd, ts=516) == 3 and call(bwd, hs=68) == 3 and call(bwd, ots=516) == 3
        assert all(call(bwd, **{k: p + 8}) == 3 for k in (views if bwd else ("q", "k", "v", "o")))
        assert _launches(call(bwd)) and _launches(call(bwd, hs=0)) and _launches(call(bwd, causal=0, prefix=p, cap=5.0, slopes=p))
        assert _launches(call(bwd, T=1, ts=0, ots=0)) and _launches(call(bwd, T=0, q=None, k=None, v=None, o=None, do=None, ws=None))
    assert _launches(call(False, lse=None))
    assert call(True, lse=None) == 1 and all(call(True, **{k: None}) == 1 for k in ("dq", "dk", "dv"))
    assert all(call(True, **{k: p + 8}) == 3 for k in ("dq", "dk", "dv"))
    assert call(True, n=256) == 9 and call(True, ws=None) == 9 and call(True, ws=p + 16) == 9


# ------------------------------------------------------- the Python calls ---

@pytest.fixture
def rec(monkeypatch):
    return host_calls.recorded(monkeypatch)


def _tensors(T=5, hq=4, hk=2, D=64):
    r = lambda *s: torch.randn(*s).to(BF16)
    i = lambda n: torch.zeros(n, dtype=I32)
    return dict(do=r(T, hq, D), q=r(T, hq, D), k=r(T, hk, D), v=r(T, hk, D), o=r(T, hq, D), lse=torch.zeros(hq, T), cu=i(4),
                prefix=i(3), slopes=torch.zeros(hq), dq=r(T, hq, D), dk=r(T, hk, D), dv=r(T, hk, D),
                ws=torch.zeros(4096, dtype=torch.uint8), st=i(1))


def _fwd(t, **kw):
    return B.olive_packed_attention_fwd(t["q"], t["k"], t["v"], t["cu"], prefix_end=t["prefix"], slopes=t["slopes"],
                                        dev_status=t["st"], out=t["o"], **kw)


def _bwd(t, **kw):
    return B.olive_packed_attention_bwd(t["do"], t["q"], t["k"], t["v"], t["o"], t["lse"], t["cu"], prefix_end=t["prefix"],
                                        slopes=t["slopes"], ws=t["ws"], dev_status=t["st"], out=(t["dq"], t["dk"], t["dv"]), **kw)


USED = {_fwd: ("q", "k", "v", "cu", "prefix", "slopes", "o", "st"),
        _bwd: ("do", "q", "k", "v", "o", "lse", "cu", "prefix", "slopes", "dq", "dk", "dv", "ws", "st")}


def test_tensors_of_another_device_type_or_shape_are_refused(rec):
    for call, names in USED.items():
        t = _tensors()
        call(t)
        made = len(rec.calls)
        for name in names:
            rec.place(t[name], 1)
            with pytest.raises(TypeError):
                call(t)
            rec.place(t[name], 0)
            if name in ("ws", "st"):
                continue
            with pytest.raises(TypeError):
                call({**t, name: t[name].to(torch.float16)})
            with pytest.raises(ValueError):
                call({**t, name: torch.cat([t[name], t[name]])})
            if t[name].dim() == 3:
                with pytest.raises(TypeError):  # the values of a head apart
                    call({**t, name: t[name].repeat_interleave(2, -1)[..., ::2]})
        assert len(rec.calls) == made


def test_views_and_forms_are_passed_on(rec):
    t = _tensors()
    qkv = torch.randn(5, 8, 64).to(BF16)
    B.olive_packed_attention_fwd(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], t["cu"])
    B.olive_packed_attention_fwd(qkv[:, :4], qkv[:, 4:5].expand(-1, 2, -1), qkv[:, 6:], t["cu"], scale=0.5, causal=False, cap=7.0)
    one, two = rec.named("olive_packed_attention_fwd")
    base = qkv.data_ptr()
    assert one[:9] == (base, 512, 64, base + 512, 512, 64, base + 768, 512, 64)
    assert one[9:20] == (4, 2, t["cu"].data_ptr(), 3, 5, 64, 0.125, 1, None, 0.0, None)
    assert two[3:6] == (base + 512, 512, 0) and two[15:20] == (0.5, 0, None, 7.0, None)


def test_gradients_that_the_backward_cannot_read_are_copied(rec):
    t = _tensors()
    q = t["q"].clone().requires_grad_()
    for g in (torch.ones(5 * 256 + 1, dtype=BF16)[1:].view(5, 4, 64), torch.ones(4, 64, dtype=BF16).expand(5, 4, 64),
              torch.ones(5, 4, 1, dtype=BF16).expand(5, 4, 64), torch.ones(5, 4, 68, dtype=BF16)[..., :64]):
        B.packed_attention(q, t["k"], t["v"], t["cu"]).backward(g)
        args = rec.named("olive_packed_attention_bwd")[-1]
        assert args[0] % 16 == 0 and args[1:3] == (256, 64)
    # (what it can read it reads)
    wide = torch.ones(5, 6, 64, dtype=BF16)
    B.packed_attention(q, t["k"], t["v"], t["cu"]).backward(wide[:, 1:5])
    assert rec.named("olive_packed_attention_bwd")[-1][:3] == (wide[:, 1:5].data_ptr(), 384, 64)
