"""One decoder layer of a student trained on packed sequences with this library's calls.

Prefixes and teacher continuations are packed (olive_splice_pack), every token gets its position in
its own sequence (olive_packed_positions), and a step runs

  embedding -> norm -> q, k, v -> heads' norm and rotation -> attention inside each sequence
  -> gated feed-forward block with the residual -> norm -> masked continuation loss

backwards through all of it, clips the gradients by their global norm and takes a plain gradient
step.  Embedding, the rows' norms, the projections and the attention are ordinary torch; the rest is
the library.  `python examples/student_layer_step.py` prints the loss and the gradients' norm of some
steps on drawn ids.
"""

from __future__ import annotations

import functools
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_36246_gb300 import binding as B  # noqa: E402

EPS = 1e-6


def rope_tables(rows, width, base=10000.0, device="cuda"):
    """cos and sin [rows, width / 2] of position times base^(-2 j / width), formed in 64 bits: at long
    positions an angle formed in 32 bits is off by more than a table entry's rounding."""
    j = torch.arange(0, width, 2, dtype=torch.float64, device=device)
    angle = torch.arange(rows, dtype=torch.float64, device=device)[:, None] * base ** (-j / width)
    return angle.cos().float(), angle.sin().float()


def init(V, d, heads, kv_heads, head_dim, f, seed=0, device="cuda"):
    """The layer's parameters, bf16 leaves.  The embedding is the LM head, transposed by lookup."""
    gen = torch.Generator(device=device).manual_seed(seed)
    w = lambda *s: (torch.randn(*s, generator=gen, device=device) / s[-1] ** 0.5).to(torch.bfloat16)
    p = dict(W=w(V, d), W_qkv=w((heads + 2 * kv_heads) * head_dim, d), W_o=w(d, heads * head_dim),
             W_gate=w(f, d), W_up=w(f, d), W_down=w(d, f))
    for name, n in (("w_q", head_dim), ("w_k", head_dim), ("w_in", d), ("w_mid", d), ("w_out", d)):
        p[name] = torch.ones(n, dtype=torch.bfloat16, device=device)
    return {k: v.requires_grad_() for k, v in p.items()}


def _rows_norm(x, w):
    f = x.float()
    return (f * (f.square().mean(-1, keepdim=True) + EPS).rsqrt() * w.float()).to(x.dtype)


def layer(p, ids, positions, sequence, tables, heads, kv_heads, qk_norm_rope=B.qk_norm_rope, gated_mlp=B.gated_mlp):
    """Hidden rows [T, d] of packed ids; `sequence` [T] numbers the tokens' sequences."""
    T, d, D = ids.numel(), p["W"].shape[1], p["w_q"].numel()
    x = p["W"][ids.long()] * d ** 0.5
    qkv = (_rows_norm(x, p["w_in"]) @ p["W_qkv"].t()).view(T, heads + 2 * kv_heads, D)
    q, k = qk_norm_rope(qkv[:, :heads], qkv[:, heads:heads + kv_heads], p["w_q"], p["w_k"], *tables, positions, EPS)
    v = qkv[:, heads + kv_heads:]
    at = torch.arange(T, device=ids.device)
    seen = (sequence[:, None] == sequence[None]) & (at[None] <= at[:, None])
    per_head = lambda t: t.transpose(0, 1).repeat_interleave(heads // t.shape[1], 0)[None]
    o = torch.nn.functional.scaled_dot_product_attention(per_head(q), per_head(k), per_head(v), attn_mask=seen)
    x = x + o[0].transpose(0, 1).reshape(T, heads * D) @ p["W_o"].t()
    x = gated_mlp(_rows_norm(x, p["w_mid"]), p["W_gate"], p["W_up"], p["W_down"], x)
    return _rows_norm(x, p["w_out"]).contiguous()


def step(p, batch, V, T, heads, kv_heads, tables, lr=0.0, max_norm=1.0, dev_status=None):
    """One training step on (prefix_ids, prefix_off, cont_ids, cont_off), all on the device: the mean
    loss of the continuation tokens and the gradients' norm before clipping, as device tensors.  What
    any call of the step, forward or backward, finds wrong on the device is in dev_status."""
    st = B.new_status() if dev_status is None else dev_status
    pk = B.olive_splice_pack(*batch, V, T, dev_status=st)
    positions = B.olive_packed_positions(pk["cu_seqlens"], T)
    sequence = (torch.arange(T, device="cuda")[:, None] >= pk["cu_seqlens"][None, 1:]).sum(1)
    hidden = layer(p, pk["ids"], positions, sequence, tables, heads, kv_heads,
                   functools.partial(B.qk_norm_rope, dev_status=st), functools.partial(B.gated_mlp, dev_status=st))
    loss = B.fused_lmhead_ce(hidden, p["W"], pk["targets"], pk["rows"], pk["n_rows"], reduction="mean", dev_status=st)
    loss.backward()
    norm = B.clip_grad_norm_(p.values(), max_norm)
    with torch.no_grad():
        for t in p.values():
            if lr:
                t -= lr * t.grad
            t.grad = None
    return loss.detach(), norm


def draw_batch(V, lens, device="cuda", seed=0):
    """A batch of (prefix, continuation) lengths with drawn ids, as device CSR arrays; and T."""
    gen = torch.Generator().manual_seed(seed)
    csr = lambda n: torch.tensor([0] + torch.tensor(n).cumsum(0).tolist(), dtype=torch.int32, device=device)
    ids = lambda n: torch.randint(0, V, (sum(n),), generator=gen, dtype=torch.int32).to(device)
    pre, con = [a for a, _ in lens], [b for _, b in lens]
    return (ids(pre), csr(pre), ids(con), csr(con)), sum(pre) + sum(con)


def main(steps=10):
    V, d, heads, kv_heads, D, f = 4096, 256, 4, 2, 64, 704
    batch, T = draw_batch(V, [(40, 88), (100, 28), (16, 112), (64, 64)])
    p = init(V, d, heads, kv_heads, D, f)
    tables = rope_tables(256, D)
    st = B.new_status()
    for i in range(steps):
        loss, norm = step(p, batch, V, T, heads, kv_heads, tables, lr=0.5, dev_status=st)
        print(f"step {i}: loss {float(loss):.4f}  gradient norm {float(norm):.4f}")
        if B.status_bits(st):
            raise SystemExit(f"step {i}: {', '.join(B.status_bits(st))}")


if __name__ == "__main__":
    main()
