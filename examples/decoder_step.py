"""A training step of one attention block and a tied output, distilled from a
teacher's top logits.

    x = E[ids] scale -> q, k, v projections -> rotary positions -> attention -> output projection
    y = x + attention's output -> logits y E^T -> divergence from the teacher's top entries

Packed sequences with padding behind them.  Everything but the products with
the weights is this library's: embed, rope, attn, distill with its gradient in
one pass, attn_grad, rope_grad, the weight gradients from 8-bit checkpoints
(act_pack, act_wgrad) and the table's by sorted tokens (embed_grad).

    python examples/decoder_step.py            # a few steps, prints the loss
"""
from __future__ import annotations

import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_19331_gb300 as iso  # noqa: E402
import synth  # noqa: E402


class Block:
    def __init__(self, vocab, heads, kv_heads, dim, dtype=torch.bfloat16, device="cuda", seed=0, pad_id=None):
        hidden = heads * dim
        shapes = [(vocab, hidden, False), ((heads + 2 * kv_heads) * dim, hidden, False), (hidden, hidden, False)]
        self.E, self.qkv, self.out = synth.base_weights(shapes, seed, device, dtype)
        self.heads, self.kv_heads, self.dim, self.pad_id = heads, kv_heads, dim, pad_id
        self.scale = hidden ** 0.5
        self.plan = iso.rope_plan(dim, base=1e6)
        self.cuts = [heads * dim, kv_heads * dim, kv_heads * dim]

    def forward(self, ids, positions, seqs):
        """(logits, what the backward pass needs)"""
        x = iso.embed(self.E, ids, scale=self.scale, pad_id=self.pad_id)
        z = x @ self.qkv.t()
        qk = z[:, :self.cuts[0] + self.cuts[1]]                  # queries and keys turn together, in place
        iso.rope(qk, positions, self.plan, out=qk)
        q, k, v = z.split(self.cuts, dim=1)
        o, lse = iso.attn(q, k, v, self.heads, self.kv_heads, seqs=seqs)
        y = x + o @ self.out.t()
        return y @ self.E.t(), (iso.act_pack(x), z, o, lse, y)

    def backward(self, ids, positions, seqs, dlogits, kept):
        """Gradients of E, the q-k-v and the output projection."""
        x_pack, z, o, lse, y = kept
        dy = dlogits @ self.E
        g_E = iso.act_wgrad(dlogits, iso.act_pack(y))
        g_out = iso.act_wgrad(dy, iso.act_pack(o))
        do = dy @ self.out
        dz = torch.zeros_like(z)                                 # (rows of no sequence stay 0)
        q, k, v = z.split(self.cuts, dim=1)
        iso.attn_grad(do, q, k, v, o, lse, self.heads, self.kv_heads, seqs=seqs, grads=dz.split(self.cuts, dim=1))
        dqk = dz[:, :self.cuts[0] + self.cuts[1]]
        iso.rope_grad(dqk, positions, self.plan, out=dqk)
        g_qkv = iso.act_wgrad(dz, x_pack)
        dx = dy + dz @ self.qkv
        iso.embed_grad(dx, ids, scale=self.scale, pad_id=self.pad_id, out=g_E, accumulate=True)
        return g_E, g_qkv, g_out

    def step(self, ids, positions, seqs, top_ids, top_logits, weights, lr=0.1):
        """One plain gradient step; returns the weighted loss before it (on the device)."""
        logits, kept = self.forward(ids, positions, seqs)
        loss, _, dlogits = iso.distill(logits, top_ids, top_logits, dloss=weights, out=logits)
        grads = self.backward(ids, positions, seqs, dlogits, kept)
        for w, g in zip((self.E, self.qkv, self.out), grads):
            w.add_(g.to(w.dtype), alpha=-lr)
        return (loss * weights).sum()


def batch(vocab, lengths, pad, top, seed=1, device="cuda"):
    """Ids, positions, offsets, the teacher's top entries and the tokens' weights of packed sequences."""
    gen = torch.Generator().manual_seed(seed)
    T = sum(lengths) + pad
    ids = torch.randint(0, vocab - 1, (T,), generator=gen)
    positions = torch.cat([torch.arange(n) for n in lengths] + [torch.zeros(pad, dtype=torch.int64)])
    seqs = torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], dtype=torch.int32)
    top_ids = torch.randint(0, vocab, (T, top), generator=gen)
    weights = torch.full((T,), 1.0 / sum(lengths))
    if pad:
        ids[T - pad:] = vocab - 1
        top_ids[T - pad:] = -1
        weights[T - pad:] = 0.0
    top_logits = 2.0 * torch.randn(T, top, generator=gen)
    return [t.to(device) for t in (ids, positions, seqs, top_ids, top_logits, weights)]


def main(steps=5):
    small = synth.QWEN["qwen1.5b"]
    vocab, dim = small["vocab"] // 8, 64
    ids, positions, seqs, top_ids, top_logits, weights = batch(vocab, [200, 150, 130], 32, 16)
    model = Block(vocab, 4, 2, dim, seed=3, pad_id=vocab - 1)
    losses = [model.step(ids, positions, seqs, top_ids, top_logits, weights) for _ in range(steps)]
    losses = torch.stack(losses).tolist()
    print(" ".join(f"{x:.4f}" for x in losses))
    return losses


if __name__ == "__main__":
    main()
