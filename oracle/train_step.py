"""Training-step operators in numpy binary64: the 8-bit activation checkpoint,
the weight gradient and the SwiGLU gradients taken from it, the token embedding
and its gradient.  Plain definitions, element by element where that is
clearest; the format's integers are exact.
"""
from __future__ import annotations

import math

import numpy as np

GROUP = 32
E_MIN = -126


def group_exponent(amax: float) -> int:
    """The least integer e >= -126 with amax <= 127 2^e."""
    if amax == 0.0:
        return E_MIN
    e = math.frexp(amax)[1] - 8          # 127 2^e < 2^(e + 7) <= amax 2^0: from below
    while amax > 127.0 * 2.0 ** e:
        e += 1
    return max(e, E_MIN)


def act_encode(x):
    """(codes int8 [T, cols up to 32], exponent bytes uint8 [T, groups]) of a matrix."""
    x = np.asarray(x, np.float64)
    T, C = x.shape
    G = -(-C // GROUP)
    v = np.zeros((T, G * GROUP))
    v[:, :C] = x
    v = v.reshape(T, G, GROUP)
    codes = np.zeros((T, G, GROUP), np.int8)
    exps = np.zeros((T, G), np.uint8)
    for t in range(T):
        for g in range(G):
            a = np.abs(v[t, g]).max()      # NaN where the group has one
            if not np.isfinite(a):
                exps[t, g] = 255
                continue
            e = group_exponent(float(a))
            exps[t, g] = e + 127
            q = np.rint(v[t, g] / 2.0 ** e)               # halves to even
            codes[t, g] = np.clip(q, -63, 63) if e == 122 else q   # 64 * 2^122 overflows binary32
    return codes.reshape(T, G * GROUP), exps


def act_decode(codes, exps, cols):
    """The values of a checkpoint."""
    T, G = exps.shape
    s = np.where(exps == 255, np.nan, np.exp2(exps.astype(np.float64) - 127.0))
    return (codes.reshape(T, G, GROUP).astype(np.float64) * s[:, :, None]).reshape(T, G * GROUP)[:, :cols]


def act_values(x):
    x = np.asarray(x, np.float64)
    return act_decode(*act_encode(x), x.shape[1])


def wgrad(dy, x_hat):
    """The gradient of y = x W^T with respect to W."""
    return np.asarray(dy, np.float64).T @ np.asarray(x_hat, np.float64)


def sigmoid(x):
    x = np.asarray(x, np.float64)
    with np.errstate(over="ignore"):
        return np.where(x >= 0, 1.0 / (1.0 + np.exp(-np.abs(x))), np.exp(-np.abs(x)) / (1.0 + np.exp(-np.abs(x))))


def swiglu(g, u):
    g = np.asarray(g, np.float64)
    return g * sigmoid(g) * u


def swiglu_grad(dh, g, u):
    """(d_gate, d_up) of h = silu(g) u."""
    g = np.asarray(g, np.float64)
    s = sigmoid(g)
    return dh * u * (s + g * s * sigmoid(-g)), dh * g * s


def embed(table, ids, scale=1.0, pad_id=-1):
    table = np.asarray(table, np.float64)
    out = np.zeros((len(ids), table.shape[1]))
    for t, i in enumerate(ids):
        if i != pad_id and 0 <= i < len(table):
            out[t] = scale * table[i]
    return out


def embed_grad(dy, ids, rows, scale=1.0, pad_id=-1):
    dy = np.asarray(dy, np.float64)
    grad = np.zeros((rows, dy.shape[1]))
    for t, i in enumerate(ids):
        if i != pad_id and 0 <= i < rows:
            grad[i] += scale * dy[t]
    return grad
