"""Embedding, rows' norm and attention as they are used: at once on streams and from threads, with
graphs that share a workspace, waits that run out, and arrays beyond 32-bit offsets."""

import os
import threading

import pytest
import torch

from paper_2609_36246_gb300 import binding as B

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def _step(lens, hq, hk, D, V, seed, **form):
    """A pass of every call on its own inputs: outputs and the status word."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(BF16)
    T, d = sum(lens), hq * D
    cu = torch.tensor([0, *torch.tensor(lens).cumsum(0).tolist()], dtype=torch.int32, device="cuda")
    ids = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    W, w, b, dy, qkv = r(V, d), r(d), r(d), r(T, d), r(T, hq + 2 * hk, D)
    q, k, v = qkv.split([hq, hk, hk], 1)
    st = B.new_status()

    def run(ws=None):
        x = B.olive_embedding_fwd(W, ids, 2.0, dev_status=st)
        y, h, stats = B.olive_row_norm_fwd(x, w, b, residual=dy, save=True)
        o, lse = B.olive_packed_attention_fwd(q, k, v, cu, dev_status=st, **form)
        grads = B.olive_packed_attention_bwd(dy.view(T, hq, D), q, k, v, o, lse, cu, ws=ws, dev_status=st, **form)
        dx, dw, db = B.olive_row_norm_bwd(dy, h, w, stats, y, ws=ws)
        dW = B.olive_embedding_bwd(dx, ids, V, 2.0, ws=ws, dev_status=st)
        return [x, y, h, stats, o, lse, *grads, dx, dw, db, dW]

    return run, st


STEPS = [lambda s: _step([900, 300, 1, 45], 8, 2, 64, 700, s), lambda s: _step([5] * 300, 4, 4, 32, 5000, s, causal=False),
         lambda s: _step([2000], 5, 1, 128, 97, s, cap=20.0)]


def _same(got, want):
    return all(torch.equal(a, b) for a, b in zip(got, want)) and len(got) == len(want)


@pytest.mark.parametrize("one", range(3))
@pytest.mark.parametrize("other", range(3))
def test_two_streams(one, other):
    steps = [STEPS[one](1), STEPS[other](2)]
    want = [run() for run, _ in steps]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in steps], [[], []]
    for _ in range(6):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(steps[i][0]())
    torch.cuda.synchronize()
    for (_, st), outs, ref in zip(steps, got, want):
        assert B.status_bits(st) == [] and all(_same(o, ref) for o in outs)


def test_two_host_threads():
    steps = [STEPS[0](3), STEPS[2](4)]
    want = [run() for run, _ in steps]
    torch.cuda.synchronize()
    got, failed = [[], []], []

    def work(i):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(8):
                    got[i].append(steps[i][0]())
            s.synchronize()
        except BaseException as e:  # (shown by the assertion below)
            failed.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    for (_, st), outs, ref in zip(steps, got, want):
        assert B.status_bits(st) == [] and len(outs) == 8 and all(_same(o, ref) for o in outs)


def test_graphs_that_share_a_workspace():
    """Two captured steps on one workspace, replayed in turn on one stream; what one leaves in it
    does not matter to the other."""
    steps = [STEPS[0](5), STEPS[1](6)]
    want = [run() for run, _ in steps]
    ws = torch.full((1 << 26,), 0xA5, dtype=torch.uint8, device="cuda")
    graphs, got = [], []
    for run, _ in steps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(run(ws))
        graphs.append(g)
    for i in (0, 1, 1, 0, 1):
        graphs[i].replay()
        assert _same(got[i], want[i])


def test_waits_that_run_out_are_reported():
    """With a limit of 0 a wait gives up when it is first looked at (a wait of some microseconds is
    over before that: so a long sequence, whose copies wait for the tiles ahead of them): a status,
    and the next call is as ever."""
    run, st = _step([16384], 8, 2, 128, 97, 7)
    want = run()
    torch.cuda.synchronize()
    old = os.environ.get("OLIVE_WAIT_LIMIT_MS")
    os.environ["OLIVE_WAIT_LIMIT_MS"] = "0"
    try:
        run()
        torch.cuda.synchronize()
    finally:
        if old is None:
            del os.environ["OLIVE_WAIT_LIMIT_MS"]
        else:
            os.environ["OLIVE_WAIT_LIMIT_MS"] = old
    assert B.status_bits(st) == ["OLIVE_ERR_TIMEOUT"]
    for _ in range(3):
        assert _same(run(), want)


def _roomy(t, stride):
    """The same values, tokens `stride` elements apart."""
    far = torch.empty(t.shape[0] * stride, dtype=t.dtype, device="cuda")
    view = far.as_strided(t.shape, (stride, t.shape[2], 1))
    view.copy_(t)
    return view


def test_attention_beyond_32_bits():
    """Tokens 2^23 elements apart: the 300th lies 2.5 G elements on."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    q, k, do = (torch.randn(300, 2, 64, generator=gen, device="cuda").to(BF16) for _ in range(3))
    cu = torch.tensor([0, 20, 300], dtype=torch.int32, device="cuda")
    o, lse = B.olive_packed_attention_fwd(q, k, k, cu)
    want = (o, lse, *B.olive_packed_attention_bwd(do, q, k, k, o, lse, cu))
    far = lambda t: _roomy(t, 1 << 23)
    fq, fo = far(q), far(torch.zeros_like(q))
    o, lse = B.olive_packed_attention_fwd(fq, k, k, cu, out=fo)
    outs = (far(torch.zeros_like(q)), torch.empty_like(k), far(torch.zeros_like(q)))
    got = (o, lse, *B.olive_packed_attention_bwd(do, fq, k, k, o, lse, cu, out=outs))
    assert _same(got, want)


def test_rows_beyond_32_bits():
    """The last rows of 2^31 + elements, against the same rows by themselves."""
    d, n = 16384, 5
    T = (1 << 31) // d + n
    x = torch.zeros(T, d, dtype=BF16, device="cuda")
    x[-n:] = torch.randn(n, d, device="cuda").to(BF16)
    x[0, 0] = 1
    w = torch.randn(d, device="cuda").to(BF16)
    y, h, stats = B.olive_row_norm_fwd(x, w, save=True)
    y0, _, stats0 = B.olive_row_norm_fwd(x[-n:].contiguous(), w, save=True)
    assert torch.equal(y[-n:], y0) and torch.equal(stats[:, -n:], stats0)
    dx, _, _ = B.olive_row_norm_bwd(x, x, w, stats, out=y)
    dx0, _, _ = B.olive_row_norm_bwd(x[-n:].contiguous(), x[-n:].contiguous(), w, stats0)
    assert torch.equal(dx[-n:], dx0)
    del y, dx, h
    # the same array as an embedding
    ids = torch.tensor([T - 1, 0, T - 2, T - 1, T], dtype=torch.int32, device="cuda")
    rows = B.olive_embedding_fwd(x, ids)
    assert torch.equal(rows[:4], x[ids[:4].long()]) and torch.isnan(rows[4]).all()
    dW = B.olive_embedding_bwd(rows, ids, T, grad_dtype=BF16, out=torch.full_like(x, 7))
    assert torch.equal(dW[T - 1], (2 * rows[0].float()).to(BF16)) and torch.equal(dW[T - 2], rows[2])
    assert torch.equal(dW[0], rows[1]) and not dW[1:T - 2].any()


def test_embedding_of_the_largest_vocabulary():
    """Every row of 2^31 - 1 is written, whatever the workspace held."""
    V, d = 2**31 - 1, 8
    ids = torch.tensor([V - 1, 0, 1 << 30, V - 1, 63], dtype=torch.int32, device="cuda")
    dy = torch.arange(1, 41, device="cuda").reshape(5, d).to(BF16)
    ws = torch.full((B.olive_workspace_size("embedding_bwd", 5, d, V),), 255, dtype=torch.uint8, device="cuda")
    dW = torch.empty((V, d), dtype=BF16, device="cuda").fill_(7)
    B.olive_embedding_bwd(dy, ids, V, ws=ws, out=dW)
    for row, tokens in ((V - 1, [0, 3]), (0, [1]), (1 << 30, [2]), (63, [4])):
        assert torch.equal(dW[row], dy[tokens].float().sum(0).to(BF16))
        dW[row] = 0
    for rows in dW.split(1 << 27):
        assert not rows.any()
