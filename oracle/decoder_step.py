"""The operators between the embedding and the loss of a training step in numpy
binary64: rotary positions, attention of one head over one sequence with its
gradients, and distillation from a teacher's top logits with its gradient.
Plain definitions.
"""
from __future__ import annotations

import numpy as np


def rope(x, positions, head_dim, freq, axis, neighbours=False, inverse=False):
    """x [T, heads * head_dim], positions [axes, T]; pair i turns by freq[i] per position on axis[i]."""
    y = np.array(x, np.float64)
    T, n = y.shape[0], len(freq)
    for h in range(y.shape[1] // head_dim):
        for i in range(n):
            a = (2 * i if neighbours else i) + h * head_dim
            b = (2 * i + 1 if neighbours else i + n) + h * head_dim
            for t in range(T):
                angle = float(positions[axis[i]][t]) * freq[i] * (-1.0 if inverse else 1.0)
                c, s = np.cos(angle), np.sin(angle)
                u, w = float(x[t, a]), float(x[t, b])
                y[t, a], y[t, b] = u * c - w * s, u * s + w * c
    return y


def sees(n, m, causal, window):
    """[n, m]: whether query i sees key j; queries stand at the keys' end."""
    i, j = np.arange(n)[:, None] + m - n, np.arange(m)[None]
    if not causal:
        return np.ones((n, m), bool)
    return (j <= i) & ((j > i - window) if window else True)


def attn(q, k, v, scale, seen):
    """(out, lse, P) of one head: queries [n, D], keys and values [m, D]."""
    n, m = seen.shape
    out, lse, P = np.zeros((n, v.shape[1])), np.full(n, -np.inf), np.zeros((n, m))
    for i in range(n):
        at = np.flatnonzero(seen[i])
        if not len(at):
            continue
        s = scale * (k[at] @ q[i])
        top = s.max()
        lse[i] = top + np.log(np.exp(s - top).sum())
        P[i, at] = np.exp(s - lse[i])
        out[i] = P[i, at] @ v[at]
    return out, lse, P


def attn_grad(dout, q, k, v, out, lse, scale, seen):
    """(dq, dk, dv) of one head from the out and lse given."""
    S = np.where(seen, scale * (q @ k.T), -np.inf)
    P = np.where(seen, np.exp(np.where(seen, S - np.where(seen.any(1), lse, 0.0)[:, None], 0.0)), 0.0)
    dS = P * (dout @ v.T - (dout * out).sum(1, keepdims=True))
    return scale * dS @ k, scale * dS.T @ q, P.T @ dout


def distill(z, ids, teacher, tau, dloss=None):
    """(loss, lse, gradient) row by row; a slot outside the vocabulary is unused."""
    T, V = z.shape
    loss, lse, grad = np.zeros(T), np.full(T, -np.inf), np.zeros((T, V))
    for t in range(T):
        x = z[t] / tau
        if V and (np.isnan(x).any() or (x == np.inf).any()):
            lse[t] = np.nan
        elif V and x.max() > -np.inf:
            lse[t] = x.max() + np.log(np.exp(x - x.max()).sum())
        used = [k for k in range(ids.shape[1]) if 0 <= ids[t, k] < V]
        w = teacher[t, used] / tau
        if not len(used) or (w == -np.inf).all():
            continue
        p = np.exp(w - w.max())
        p /= p.sum()
        with np.errstate(invalid="ignore"):
            for pk, k in zip(p, used):
                if pk != 0.0:
                    loss[t] += tau ** 2 * pk * (np.log(pk) - (x[ids[t, k]] - lse[t]))
            grad[t] = np.exp(x - lse[t])
            for pk, k in zip(p, used):
                grad[t, ids[t, k]] -= pk
            if dloss is not None:
                grad[t] *= dloss[t] * tau
    return loss, lse, grad
