"""Calls in flight at once, on two streams and from two host threads.

Cut tiles of the gated block wait for other CTAs of their own launch, and a launch starts under the one
ahead of it: neither may depend on having the GPU to itself.  Every wait is bounded, so a launch that
could not go on would end with a status and wrong bits, not hang.
"""

import threading

import pytest
import torch

from paper_2609_36246_gb300 import binding as B

pytestmark = pytest.mark.gpu

# shapes whose tiles are cut in two and in many pieces, ones dealt whole, and few rows by clusters
SHAPES = [(138, 256, 12200), (512, 2048, 6144), (900, 1024, 1408), (12, 2048, 768), (64, 4096, 512)]


def _step(T, d, f, seed):
    """A step of every call of the layer on its own inputs: outputs and the status word."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)
    x, res, dy, w = r(T, d), r(T, d), r(T, d), (r(f, d) * d ** -0.5, r(f, d) * d ** -0.5, r(d, f) * 0.05)
    q, k, wq = r(T, 6, 64), r(T, 2, 64), r(64)
    table = torch.rand(T, 32, generator=gen, device="cuda")
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    st = B.new_status()

    def run():
        y, saved = B.olive_gated_mlp_fwd(x, *w, residual=res, save=True, dev_status=st)
        grads = B.olive_gated_mlp_bwd(dy, x, *w, saved, dev_status=st)
        heads = B.olive_qk_norm_rope_bwd(q, k, q, k, wq, wq, table, table, pos, dev_status=st)
        out = [torch.empty_like(g) for g in grads]
        return [y, saved, *grads, *heads, B.olive_grad_clip(grads, 0.1, out=out), *out]

    return run, st


def _same(got, want):
    return all(torch.equal(a, b) for a, b in zip(got, want)) and len(got) == len(want)


@pytest.mark.parametrize("one", SHAPES)
@pytest.mark.parametrize("other", SHAPES[:3])
def test_two_streams(one, other):
    steps = [_step(*one, seed=1), _step(*other, seed=2)]
    want = [run() for run, _ in steps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    got = [[], []]
    for _ in range(8):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(steps[i][0]())
    torch.cuda.synchronize()
    for (_, st), outs, ref in zip(steps, got, want):
        assert B.status_bits(st) == [] and all(_same(o, ref) for o in outs)


def test_two_host_threads():
    steps = [_step(*SHAPES[1], seed=3), _step(*SHAPES[0], seed=4)]
    want = [run() for run, _ in steps]
    torch.cuda.synchronize()
    got, failed = [[], []], []

    def work(i):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(12):
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
        assert B.status_bits(st) == [] and len(outs) == 12 and all(_same(o, ref) for o in outs)
