"""Pins of oracle/decoder_step.py: by hand, by invariants and by differences."""
import numpy as np
import pytest

from oracle import decoder_step as R


def _difference(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        d = np.zeros_like(x)
        d[i] = h
        g[i] = (f(x + d) - f(x - d)) / (2 * h)
    return g


@pytest.mark.parametrize("neighbours", [False, True])
def test_rope_by_complex_numbers_and_back(neighbours):
    rng = np.random.default_rng(0)
    x, p = rng.normal(size=(5, 2 * 10)), np.array([[0, 1, -3, 70, 100000], [5, 5, 6, 7, 8]])
    freq, axis = [1.0, 0.3, 1e-3], [0, 1, 0]
    y = R.rope(x, p, 10, freq, axis, neighbours)
    for h in range(2):
        v = x[:, h * 10:(h + 1) * 10]
        first = v[:, 0:6:2] if neighbours else v[:, :3]
        second = v[:, 1:6:2] if neighbours else v[:, 3:6]
        w = (first + 1j * second) * np.exp(1j * p[axis].T * np.array(freq))
        got = y[:, h * 10:(h + 1) * 10]
        assert np.allclose(got[:, 0:6:2] if neighbours else got[:, :3], w.real, atol=1e-9)
        assert np.allclose(got[:, 1:6:2] if neighbours else got[:, 3:6], w.imag, atol=1e-9)
        assert np.array_equal(got[:, 6:], v[:, 6:])
    assert np.allclose(R.rope(y, p, 10, freq, axis, neighbours, inverse=True), x, atol=1e-12)
    dy = rng.normal(size=y.shape)
    dx = _difference(lambda a: (R.rope(a, p, 10, freq, axis, neighbours) * dy).sum(), x)
    assert np.allclose(R.rope(dy, p, 10, freq, axis, neighbours, inverse=True), dx, atol=1e-7)


@pytest.mark.parametrize("n,m,causal,window", [(4, 4, True, 0), (3, 6, True, 2), (5, 3, True, 0), (3, 4, False, 0)])
def test_attention_and_its_gradients(n, m, causal, window):
    rng = np.random.default_rng(1)
    q, k, v, do = (rng.normal(size=s) for s in ((n, 3), (m, 3), (m, 3), (n, 3)))
    seen = R.sees(n, m, causal, window)
    for i in range(n):
        for j in range(m):
            at = i + m - n
            assert seen[i, j] == (not causal or (j <= at and (not window or j > at - window)))
    out, lse, P = R.attn(q, k, v, 0.7, seen)
    live = seen.any(1)
    assert np.allclose(P.sum(1), live) and (out[~live] == 0).all() and (lse[~live] == -np.inf).all()

    def value(q, k, v):
        return (R.attn(q, k, v, 0.7, seen)[0] * do).sum()
    dq, dk, dv = R.attn_grad(do, q, k, v, out, lse, 0.7, seen)
    assert np.allclose(dq, _difference(lambda a: value(a, k, v), q), atol=1e-7)
    assert np.allclose(dk, _difference(lambda a: value(q, a, v), k), atol=1e-7)
    assert np.allclose(dv, _difference(lambda a: value(q, k, a), v), atol=1e-7)


def test_distillation_by_definition_and_by_differences():
    rng = np.random.default_rng(2)
    z, t = rng.normal(size=(3, 7)), rng.normal(size=(3, 4))
    ids, tau, g = np.array([[0, 3, 3, -1], [6, 5, 4, 2], [-1, -1, -1, -1]]), 1.7, np.array([0.3, -2.0, 5.0])
    loss, lse, grad = R.distill(z, ids, t, tau, g)
    assert np.allclose(lse, np.log(np.exp(z / tau).sum(1)))
    # row 1 uses every slot: tau^2 times the divergence of two distributions
    p = np.exp(t[1] / tau) / np.exp(t[1] / tau).sum()
    logq = z[1] / tau - lse[1]
    assert np.isclose(loss[1], tau ** 2 * (p * (np.log(p) - logq[ids[1]])).sum())
    assert loss[2] == 0 and (grad[2] == 0).all()
    assert np.allclose(grad, _difference(lambda a: (R.distill(a, ids, t, tau)[0] * g).sum(), z), atol=1e-6)
    # one slot: the cross-entropy
    loss, lse, grad = R.distill(z, ids[:, 1:2], t[:, 1:2], 1.0, np.ones(3))
    assert np.isclose(loss[0], lse[0] - z[0, 3])
