"""What the Python entry points of the layer's calls decide by themselves, on the host (host_calls.py):
nothing here launches a kernel."""

import array
import random

import pytest
import torch

from paper_2609_36246_gb300 import binding as B
from tests import host_calls

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture
def rec(monkeypatch):
    return host_calls.recorded(monkeypatch)


def _mlp(T=4, d=64, f=72):
    r = lambda *s: torch.randn(*s).to(BF16)
    return dict(x=r(T, d), W_gate=r(f, d), W_up=r(f, d), W_down=r(d, f), residual=r(T, d), dy=r(T, d),
                saved=torch.zeros(2, T, f, dtype=torch.int16))


def _qk(T=5, hq=3, hk=2, D=64, R=64, dtype=BF16):
    r = lambda *s: torch.randn(*s).to(dtype)
    return dict(q=r(T, hq, D), k=r(T, hk, D), w_q=r(D), w_k=r(D), cos=torch.ones(9, R // 2), sin=torch.zeros(9, R // 2),
                positions=torch.arange(T, dtype=torch.int32), g_q=r(T, hq, D), g_k=r(T, hk, D))


def _extra():
    """A workspace and a status word of the caller's."""
    return dict(ws=torch.zeros(4096, dtype=torch.uint8), dev_status=torch.zeros(1, dtype=torch.int32))


def _like_outputs(s, *names):
    return {"out%d" % i: torch.empty_like(s[n]) for i, n in enumerate(names)}


# each call as (its tensors, the call of them): every tensor of it in turn is on another device
def _calls():
    s, e = _mlp(), _extra()
    yield {**{k: s[k] for k in ("x", "W_gate", "W_up", "W_down", "residual")}, **_like_outputs(s, "x"), **e}, lambda t: \
        B.olive_gated_mlp_fwd(t["x"], t["W_gate"], t["W_up"], t["W_down"], t["residual"], ws=t["ws"],
                              dev_status=t["dev_status"], out=t["out0"])
    s, e = _mlp(), _extra()
    weights = ("W_gate", "W_up", "W_down")
    yield {**{k: v for k, v in s.items() if k != "residual"}, **_like_outputs(s, "x", *weights), **e}, lambda t: \
        B.olive_gated_mlp_bwd(t["dy"], t["x"], *(t[n] for n in weights), t["saved"], ws=t["ws"],
                              dev_status=t["dev_status"], out=[t["out%d" % i] for i in range(4)])
    names = ("q", "k", "w_q", "w_k", "cos", "sin", "positions")
    s, e = _qk(), _extra()
    yield {**{k: s[k] for k in names}, **_like_outputs(s, "q", "k"), "dev_status": e["dev_status"]}, lambda t: \
        B.olive_qk_norm_rope_fwd(*(t[n] for n in names), dev_status=t["dev_status"], out=(t["out0"], t["out1"]))
    s, e = _qk(), _extra()
    yield {**s, **_like_outputs(s, "q", "k"), **e}, lambda t: \
        B.olive_qk_norm_rope_bwd(t["g_q"], t["g_k"], *(t[n] for n in names), ws=t["ws"], dev_status=t["dev_status"],
                                 out=(t["out0"], t["out1"]))
    yield dict(cu=torch.zeros(3, dtype=torch.int32), out=torch.zeros(7, dtype=torch.int32)), lambda t: \
        B.olive_packed_positions(t["cu"], 7, out=t["out"])
    yield dict(g=torch.ones(5), h=torch.ones(6), a=torch.ones(5), b=torch.ones(6), norm=torch.ones(1), ws=_extra()["ws"]), \
        lambda t: B.olive_grad_clip([t["g"], t["h"]], 1.0, out=[t["a"], t["b"]], norm=t["norm"], ws=t["ws"])


def test_tensors_of_another_device_are_refused(rec):
    for tensors, call in _calls():
        call(tensors)
        made = len(rec.calls)
        for name, t in tensors.items():
            rec.place(t, 1)
            with pytest.raises(TypeError):
                call(tensors)
            rec.place(t, 0)
        # (all of them elsewhere: the launch would still go to the current device)
        for t in tensors.values():
            rec.place(t, 1)
        with pytest.raises(TypeError):
            call(tensors)
        assert len(rec.calls) == made


def test_calls_before_them_refuse_it_too(rec):
    h, W = torch.zeros(4, 64, dtype=BF16), torch.zeros(50, 64, dtype=BF16)
    ids = [torch.zeros(4, dtype=torch.int32) for _ in range(3)]
    run = lambda: B.olive_token_logprob_fwd(h, W, *ids)
    run()
    made = len(rec.calls)
    for t in (h, W, *ids):
        rec.place(t, 1)
        with pytest.raises(TypeError):
            run()
        rec.place(t, 0)
    assert len(rec.named("olive_token_logprob_fwd")) == 1 and len(rec.calls) == made


def _pieces(flat, *spans):
    return [flat[a:b] for a, b in spans]


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gradients_that_share_memory_are_not_scaled(rec, dtype):
    flat, other = torch.ones(100, dtype=dtype), torch.ones(100, dtype=dtype)
    clip = lambda g, **k: B.olive_grad_clip(g, 1.0, **k)
    same = [flat, other, flat]
    for g in (same, [flat[:10], flat[9:20]], [flat[50:60], other, flat[:100]], [flat, other[:5], flat[99:]]):
        with pytest.raises(ValueError):
            clip(g)
        with pytest.raises(ValueError):  # the outputs
            clip([torch.ones(t.numel(), dtype=dtype) for t in g], out=g)
        fresh = [torch.empty_like(t) for t in g]
        clip(g, out=fresh)  # read only: nothing is written twice
        clip(g, out=None)
    # an output over another gradient, and over its own but for an element
    with pytest.raises(ValueError):
        clip([flat, other], out=[other, flat])
    with pytest.raises(ValueError):
        clip([flat[:50]], out=[flat[1:51]])
    with pytest.raises(ValueError):
        clip([flat, flat, other], out=[torch.empty_like(flat), torch.empty_like(flat), flat])
    assert len(rec.named("olive_grad_clip")) == 8


def test_gradients_that_only_touch_are_scaled(rec):
    flat, other = torch.ones(100), torch.ones(100, dtype=BF16)
    g = _pieces(flat, (50, 100), (0, 25), (25, 50)) + _pieces(other, (1, 3), (0, 1), (3, 100))
    empty = [flat[10:10], other[:0], flat[100:], torch.ones(0)]
    for some in (g, g + empty, empty, [flat, other] + empty, []):
        B.olive_grad_clip(some, 1.0)
        B.olive_grad_clip(some, 1.0, out=[t.clone() for t in some])
        B.olive_grad_clip(some, 1.0, out=[t if i % 2 else t.clone() for i, t in enumerate(some)])
    assert len(rec.named("olive_grad_clip")) == 15


def test_one_parameter_is_clipped(rec):
    """Not its rows, which hold no gradient."""
    p = torch.nn.Parameter(torch.zeros(4, 3))
    p.grad = torch.ones(4, 3)
    B.clip_grad_norm_(p, 1.0)
    B.clip_grad_norm_([p], 1.0)
    one, listed = rec.named("olive_grad_clip")
    assert one[4] == listed[4] == 1
    p.grad = None
    B.clip_grad_norm_(p, 1.0)
    assert rec.named("olive_grad_clip")[-1][4] == 0


def test_a_tied_parameter_is_clipped_once(rec):
    p, q = (torch.nn.Parameter(torch.zeros(5)) for _ in range(2))
    p.grad, q.grad = torch.ones(5), torch.ones(5)
    for listed in ([p, q, p], [p, p], [q, p]):
        B.clip_grad_norm_(listed, 1.0)
    assert [a[4] for a in rec.named("olive_grad_clip")] == [2, 1, 2]
    q.grad = p.grad  # one gradient held by two parameters
    B.clip_grad_norm_([p, q], 1.0)
    assert rec.named("olive_grad_clip")[-1][4] == 1


def test_gradients_in_other_orders_are_clipped(rec, monkeypatch):
    """A transposed gradient is taken as it lies; one with gaps through a copy that goes back."""
    p = [torch.nn.Parameter(torch.zeros(6, 4)) for _ in range(3)]
    p[0].grad = torch.arange(24.0).view(4, 6).t()
    wide = torch.arange(48.0).view(6, 8)
    p[1].grad = wide[:, ::2]
    p[2].grad = torch.ones(6, 4)
    seen = []
    monkeypatch.setattr(B, "olive_grad_clip", lambda g, limit: seen.extend(g) or [t.mul_(0.5) for t in g] and "norm")
    assert B.clip_grad_norm_(p, 1.0) == "norm"
    assert all(t.is_contiguous() for t in seen) and seen[0].data_ptr() == p[0].grad.data_ptr() and seen[2] is p[2].grad
    assert torch.equal(p[0].grad, torch.arange(24.0).view(4, 6).t() / 2)
    assert torch.equal(p[1].grad, torch.arange(48.0).view(6, 8)[:, ::2] / 2)
    assert torch.equal(wide[:, 1::2], torch.arange(48.0).view(6, 8)[:, 1::2])


def _second_order(out, leaf):
    """Differentiates a gradient: what a penalty on it does."""
    g, = torch.autograd.grad(out.float().square().sum(), [leaf], create_graph=True)
    (out.float().sum() + g.float().square().sum()).backward()


def test_second_derivatives_of_the_layer_are_refused(rec):
    """They are not formed; leaving them out unsaid would give a wrong gradient."""
    s = _mlp()
    for leaf in ("x", "W_gate"):
        t = {k: v.clone().requires_grad_(k == leaf) for k, v in s.items() if k not in ("dy", "saved")}
        with pytest.raises(RuntimeError, match="once_differentiable"):
            _second_order(B.gated_mlp(*t.values()), t[leaf])
    s = _qk()
    for leaf in ("q", "w_k"):
        t = {k: v.clone().requires_grad_(k == leaf) for k, v in s.items() if not k.startswith("g_")}
        with pytest.raises(RuntimeError, match="once_differentiable"):
            _second_order(sum(y.float().sum() for y in B.qk_norm_rope(*t.values())), t[leaf])


@pytest.mark.parametrize("others", [(), ("x", "W_down")])
def test_second_derivatives_of_the_residual(rec, others):
    """Its gradient is the output's: (sum y + sum (2 y)^2) differentiates to 1 + 8 y, with y = 1."""
    t = {k: v.clone().requires_grad_(k == "residual" or k in others) for k, v in _mlp().items() if k not in ("dy", "saved")}
    _second_order(B.gated_mlp(*t.values()), t["residual"])
    assert torch.equal(t["residual"].grad, torch.full_like(t["residual"], 9.0))


@pytest.mark.parametrize("single_pass", [True, False])
def test_second_derivatives_of_the_loss_are_refused(rec, single_pass):
    ids = [torch.zeros(4, dtype=torch.int32) for _ in range(3)]
    h, W = torch.zeros(4, 64, dtype=BF16, requires_grad=True), torch.zeros(50, 64, dtype=BF16, requires_grad=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        _second_order(B.fused_lmhead_ce(h, W, *ids, single_pass=single_pass), h)


def test_autograd_forms_pass_the_status_word_on(rec):
    """To the forward's call and to the backward's."""
    st = torch.zeros(1, dtype=torch.int32)
    s = _mlp()
    B.gated_mlp(*(s[k].requires_grad_() for k in ("x", "W_gate", "W_up", "W_down", "residual")), dev_status=st).sum().backward()
    s = _qk()
    leaf = [s[k].requires_grad_(s[k].dtype == BF16) for k in ("q", "k", "w_q", "w_k", "cos", "sin", "positions")]
    sum(y.sum() for y in B.qk_norm_rope(*leaf, dev_status=st)).backward()
    for single_pass in (True, False):
        h, W = torch.zeros(4, 64, dtype=BF16, requires_grad=True), torch.zeros(50, 64, dtype=BF16, requires_grad=True)
        ids = [torch.zeros(4, dtype=torch.int32) for _ in range(3)]
        B.fused_lmhead_ce(h, W, *ids, single_pass=single_pass, dev_status=st).backward()
    with torch.no_grad():
        B.gated_mlp(*list(_mlp().values())[:4], dev_status=st)
    names = [c.name for c in rec.calls]
    for name, times in (("olive_gated_mlp_fwd", 2), ("olive_gated_mlp_bwd", 1), ("olive_qk_norm_rope_fwd", 1),
                        ("olive_qk_norm_rope_bwd", 1), ("olive_token_loss_fwd_bwd", 1), ("olive_token_logprob_fwd", 1),
                        ("olive_token_loss_bwd", 1)):
        assert names.count(name) == times, name
        assert all(args[-2] == st.data_ptr() for args in rec.named(name)), name  # (the stream is last)


def test_nothing_is_saved_without_gradients(rec):
    """Parameters ask for gradients also where autograd is off."""
    s = _mlp()
    leaf = [torch.nn.Parameter(s[k]) for k in ("W_gate", "W_up", "W_down")]
    saved = lambda: rec.named("olive_gated_mlp_fwd")[-1][10]
    B.gated_mlp(s["x"], *leaf)
    assert saved() is not None
    for off in (torch.no_grad, torch.inference_mode):
        with off():
            y = B.gated_mlp(s["x"], *leaf, s["residual"], "gelu_tanh")
        assert saved() is None and not y.requires_grad
        assert rec.named("olive_gated_mlp_fwd")[-1][4] == s["residual"].data_ptr()
        assert rec.named("olive_gated_mlp_fwd")[-1][8] == B.ACT["gelu_tanh"]
    B.gated_mlp(*(s[k] for k in ("x", "W_gate", "W_up", "W_down")), s["residual"].requires_grad_())
    assert saved() is None


def _cat_loss(parts):
    """Parts side by side and a sum that weighs them differently: their gradients are views."""
    y = torch.cat(parts, -1).float()
    return (y * torch.arange(1, y.numel() + 1).view(y.shape)).sum()


@pytest.mark.parametrize("D", [8, 64])
@pytest.mark.parametrize("before,after", [(0, 4), (4, 0), (3, 1), (8, 8), (0, 0)])
def test_gradients_that_autograd_hands_over_as_views(rec, D, before, after):
    """What lies off the 16-byte rule is copied, what fits is read where it is."""
    s = _qk(D=D, R=8)
    yq, yk = B.qk_norm_rope(*(s[k].requires_grad_(k in "qk") for k in ("q", "k", "w_q", "w_k", "cos", "sin", "positions")))
    pad = lambda y, n: [torch.zeros(*y.shape[:2], n, dtype=y.dtype)] if n else []
    (_cat_loss(pad(yq, before) + [yq] + pad(yq, after)) + _cat_loss(pad(yk, before) + [yk] + pad(yk, after))).backward()
    gq, gq_t, gq_h, gk, gk_t, gk_h = rec.named("olive_qk_norm_rope_bwd")[0][:6]
    assert gq % 16 == 0 and gk % 16 == 0 and not any(x % 8 for x in (gq_t, gq_h, gk_t, gk_h))
    assert gq_h == (D if before % 8 or after % 8 else D + before + after)


@pytest.mark.parametrize("T", [4, 1])
def test_output_gradients_that_start_anywhere(rec, T):
    s = _mlp(T=T)
    y = B.gated_mlp(s["x"].requires_grad_(), *(s[k] for k in ("W_gate", "W_up", "W_down")))
    off = torch.zeros(T * 64 + 3, dtype=BF16)[3:].view(T, 64)
    assert off.is_contiguous() and off.data_ptr() % 16 == 6
    y.backward(off)
    assert rec.named("olive_gated_mlp_bwd")[0][0] % 16 == 0


def test_drawn_lists_against_all_pairs(rec):
    """olive_grad_clip_apart against every pair of spans, with and without shared sources."""
    rng = random.Random(1)
    share = lambda a, m, b, n: m > 0 and n > 0 and a < b + n and b < a + m
    seen = [0, 0]
    for trial in range(20000):
        n = rng.randint(0, 5) if trial % 100 else 130 + trial // 200
        room = 30 if n < 10 else 40 * n
        num, kind = [rng.randint(0, 3) for _ in range(n)], [rng.randint(0, 1) for _ in range(n)]
        dst = [64 + 4 * rng.randint(0, room) for _ in range(n)]
        src = [d if rng.random() < 0.5 else 64 + 4 * rng.randint(0, room) for d in dst]
        size = [c * (4 if k else 2) for c, k in zip(num, kind)]
        apart = not any(share(dst[i], size[i], dst[j], size[j]) or share(src[j], size[j], dst[i], size[i])
                        for i in range(n) for j in range(n) if i != j)
        apart = apart and not any(s != d and share(s, m, d, m) for s, d, m in zip(src, dst, size))
        table = array.array("Q", src + dst + num)
        at, kinds = table.buffer_info()[0], array.array("i", kind)
        got = rec.olive_grad_clip_apart(at, at + 8 * n, at + 16 * n, kinds.buffer_info()[0], n)
        assert got == (0 if apart else 1), (src, dst, num, kind)
        assert rec.olive_grad_clip_apart(at, None, at + 16 * n, kinds.buffer_info()[0], n) == 0
        seen[apart] += 1
    assert min(seen) > 2000


def test_refusals_of_the_list_check(rec):
    some = array.array("q", [0, 1 << 20, 4, 0])
    at = some.buffer_info()[0]
    check = rec.olive_grad_clip_apart
    assert check(at, at, at, at, -1) == 2 and check(None, None, None, None, 0) == 0
    assert check(None, at, at, at, 1) == 1 and check(at, at, None, at, 1) == 1 and check(at, at, at, None, 1) == 1


def test_host_tensors_are_refused_with_a_name_also_without_a_gpu():
    s, q = _mlp(), _qk()
    with pytest.raises(TypeError, match="x must"):
        B.olive_gated_mlp_fwd(*list(s.values())[:4])
    with pytest.raises(TypeError, match="q and k must"):
        B.olive_qk_norm_rope_fwd(*list(q.values())[:7])
    with pytest.raises(TypeError, match="cu_seqlens must"):
        B.olive_packed_positions(torch.zeros(3, dtype=torch.int32), 4)
