"""The example's training step (pack, positions, heads' norm and rotation, gated block, loss, clipping)
against the same layer in 64 bits.

Tolerances.  Hidden rows pass through about ten bf16 roundings in series (half a last place each,
2^-8 at most and 2^-8 / sqrt(3) in the mean square): the loss, a mean over some hundred tokens of
log-probs that move with the hidden rows, is allowed 1 %, the gradients' norm 2 %.  Each gradient
adds the backward pass's roundings, as many again: 5 % in the norm.
"""

import pytest
import torch

from examples import student_layer_step as E

pytestmark = pytest.mark.gpu

V, D_MODEL, HEADS, KV, D, F = 1000, 128, 4, 2, 64, 328
LENS = [(5, 20), (33, 1), (1, 40), (12, 30)]


def _plain_qk(q, k, w_q, w_k, cos, sin, positions, eps):
    c, s = (t.double()[positions.long()][:, None] for t in (cos, sin))
    out = []
    for x, w in ((q, w_q), (k, w_k)):
        n = w * x / (x.square().mean(-1, keepdim=True) + eps).sqrt()
        a, b = n.chunk(2, -1)
        out.append(torch.cat((a * c - b * s, b * c + a * s), -1))
    return out


def _plain_mlp(x, wg, wu, wd, residual):
    return (torch.nn.functional.silu(x @ wg.t()) * (x @ wu.t())) @ wd.t() + residual


def _reference(p, batch, T, tables):
    """Loss, gradients and their norm in 64 bits, from the definitions."""
    pre, po, con, co = [t.cpu().tolist() for t in batch]
    ids, pos, seq, rows, targets = [], [], [], [], []
    for i in range(len(po) - 1):
        a, b = pre[po[i]:po[i + 1]], con[co[i]:co[i + 1]]
        start = len(ids)
        ids += a + b
        pos += range(len(a) + len(b))
        seq += [i] * (len(a) + len(b))
        rows += range(start + len(a) - 1, start + len(a) + len(b) - 1)
        targets += b
    cuda = lambda t: torch.tensor(t, device="cuda")
    q = {k: v.detach().double().requires_grad_() for k, v in p.items()}
    real_norm = E._rows_norm
    E._rows_norm = lambda x, w: w * x * (x.square().mean(-1, keepdim=True) + E.EPS).rsqrt()
    try:
        hidden = E.layer(q, cuda(ids), cuda(pos), cuda(seq), tables, HEADS, KV, _plain_qk, _plain_mlp)
    finally:
        E._rows_norm = real_norm
    loss = torch.nn.functional.cross_entropy(hidden[cuda(rows)] @ q["W"].t(), cuda(targets))
    loss.backward()
    grads = {k: v.grad for k, v in q.items()}
    return float(loss.detach()), grads, float(sum(g.square().sum() for g in grads.values()) ** 0.5)


def test_step_against_64_bits():
    batch, T = E.draw_batch(V, LENS)
    p = E.init(V, D_MODEL, HEADS, KV, D, F)
    tables = E.rope_tables(64, D)
    ref, grads, ref_norm = _reference(p, batch, T, tables)
    seen = {}
    for name, t in p.items():
        t.register_hook(lambda g, name=name: seen.__setitem__(name, seen[name] + g if name in seen else g))
    loss, norm = E.step(p, batch, V, T, HEADS, KV, tables)
    assert abs(float(loss) - ref) <= 0.01 * ref and abs(float(norm) - ref_norm) <= 0.02 * ref_norm
    for name, g in grads.items():
        got = seen[name].double()
        assert float((got - g).norm()) <= 0.05 * float(g.norm()), (name, float((got - g).norm() / g.norm()))


def test_steps_lower_the_loss():
    batch, T = E.draw_batch(V, LENS, seed=3)
    p = E.init(V, D_MODEL, HEADS, KV, D, F, seed=1)
    tables = E.rope_tables(64, D)
    losses = [float(E.step(p, batch, V, T, HEADS, KV, tables, lr=0.5)[0]) for _ in range(12)]
    assert losses[-1] < 0.8 * losses[0], losses
