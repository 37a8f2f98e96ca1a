"""Training steps of a token embedding and one SwiGLU block under ISO[AdamW].

    ids -> E[ids] scale -> gate, up projections -> silu(gate) up -> down projection -> loss

The forward pass keeps its activations as 8-bit checkpoints (act_pack,
swiglu_pack); the backward pass takes the SwiGLU gradients and every weight
gradient from them (swiglu_grad, act_wgrad) and the table's gradient by sorted
tokens (embed_grad).  Each projection then takes one fixed-spectrum step on its
frames (opt_step); the table takes a plain gradient step.  Projections'
products with their weights are torch's.

    python examples/mlp_step.py            # 20 steps, prints the loss
"""
from __future__ import annotations

import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_19331_gb300 as iso  # noqa: E402
import synth  # noqa: E402


class Projection:
    """W (out x in) = U S V^T with its frames and AdamW moments."""

    def __init__(self, W: torch.Tensor):
        self.W = W
        self.U, self.S, Vt = iso.thin_svd(W)
        self.V = Vt.t().contiguous()
        self.moments = [torch.zeros(f.shape, dtype=torch.float32, device=W.device)
                        for f in (self.U, self.U, self.V, self.V)]

    def step(self, grad, lr, t):
        iso.opt_step(self.U, self.V, self.S, grad, *self.moments, self.W, W_out=self.W, lr=lr, step=t)


class Block:
    def __init__(self, vocab, hidden, inter, dtype=torch.bfloat16, device="cuda", seed=0, pad_id=None):
        shapes = [(vocab, hidden, False), (2 * inter, hidden, False), (hidden, inter, False)]
        E, gate_up, down = synth.base_weights(shapes, seed, device, dtype)
        self.E, self.scale, self.pad_id, self.inter = E, hidden ** 0.5, pad_id, inter
        self.gate_up, self.down = Projection(gate_up), Projection(down)
        self.t = 0

    def forward(self, ids):
        """(y, what the backward pass needs): activations leave as 8-bit checkpoints."""
        x = iso.embed(self.E, ids, scale=self.scale, pad_id=self.pad_id)
        x_pack = iso.act_pack(x)
        z = x @ self.gate_up.W.t()
        h, gate_pack, up_pack = iso.swiglu_pack(z[:, :self.inter], z[:, self.inter:])
        return h @ self.down.W.t(), (x_pack, gate_pack, up_pack)

    def backward(self, ids, dy, kept):
        """Gradients of E, the gate-up and the down projection."""
        x_pack, gate_pack, up_pack = kept
        dh = dy @ self.down.W
        dz = torch.empty(len(dy), 2 * self.inter, dtype=dy.dtype, device=dy.device)
        h = torch.empty_like(dh)
        iso.swiglu_grad(dh, gate_pack, up_pack, out=(dz[:, :self.inter], dz[:, self.inter:], h))
        g_down = iso.act_wgrad(dy, iso.act_pack(h))
        g_gate_up = iso.act_wgrad(dz, x_pack)
        g_E = iso.embed_grad(dz @ self.gate_up.W, ids, self.E.shape[0], scale=self.scale, pad_id=self.pad_id)
        return g_E, g_gate_up, g_down

    def step(self, ids, target, lr=1e-3, lr_embed=0.1):
        """One training step on the mean squared error; returns the loss before it (on the device)."""
        y, kept = self.forward(ids)
        diff = y.float() - target
        g_E, g_gate_up, g_down = self.backward(ids, (diff * (2.0 / diff.numel())).to(y.dtype), kept)
        self.t += 1
        self.gate_up.step(g_gate_up, lr, self.t)
        self.down.step(g_down, lr, self.t)
        self.E.add_(g_E.to(self.E.dtype), alpha=-lr_embed)
        return diff.square().mean()


def main(steps=20, tokens=512):
    small = synth.QWEN["qwen1.5b"]
    vocab, hidden, inter = small["vocab"] // 8, small["hidden"] // 8, small["inter"] // 8
    gen = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
    target = Block(vocab, hidden, inter, dtype=torch.float32, seed=2).forward(ids)[0]
    model = Block(vocab, hidden, inter, dtype=torch.float32, seed=3)
    losses = [model.step(ids, target) for _ in range(steps)]
    losses = torch.stack(losses).tolist()
    print(" ".join(f"{x:.3e}" for x in losses))
    return losses


if __name__ == "__main__":
    main()
