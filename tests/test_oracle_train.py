"""Pins of the training-step oracle (oracle/train_step.py): the checkpoint
format against its definition, the gradients against central differences."""
import math

import numpy as np
import pytest

from oracle import train_step as R


def _rng(seed):
    return np.random.default_rng(seed)


def test_group_exponent_is_the_least_that_fits():
    cases = [127.0 * 2.0 ** k for k in range(-130, 121, 7)]
    cases += [np.nextafter(np.float32(c), np.float32(np.inf)) for c in cases] + [1.0, 0.5, 63.5, 64.0, 3e38, 1e-45]
    for a in map(float, cases):
        e = R.group_exponent(a)
        assert a <= 127.0 * 2.0 ** e and e >= R.E_MIN
        assert e == R.E_MIN or a > 127.0 * 2.0 ** (e - 1)


def test_checkpoint_hand_worked():
    x = np.zeros((1, 33))
    x[0, :4] = [127.0, 0.5, 1.5, -2.5]       # e = 0: halves to even
    x[0, 32] = 63.75                          # second group, e = -1: 127.5 > 127, so e = 0
    codes, exps = R.act_encode(x)
    assert exps.tolist() == [[127, 127]]
    assert codes[0, :4].tolist() == [127, 0, 2, -2] and codes[0, 32] == 64 and not codes[0, 33:].any()
    assert R.act_values(x)[0, 32] == 64.0


def test_checkpoint_error_and_exactness():
    x = _rng(1).normal(size=(64, 96)) * np.exp(_rng(2).normal(size=(64, 1)) * 4)
    v = R.act_values(x)
    a = np.abs(x.reshape(64, 3, 32)).max(2, keepdims=True)
    step = 2.0 ** np.vectorize(R.group_exponent)(a)
    assert (np.abs(v - x).reshape(64, 3, 32) <= step / 2).all() and (step <= 2 * a / 127).all()
    # bfloat16 holds every value: eight significant bits
    m, _ = np.frexp(v)
    assert (m * 256 == np.rint(m * 256)).all()
    # packing the values again changes nothing where a group keeps its exponent
    w = R.act_values(v)
    assert np.array_equal(w, v)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_non_finite_group_stands_for_nan(bad):
    x = np.ones((2, 64))
    x[1, 40] = bad
    v = R.act_values(x)
    assert np.isnan(v[1, 32:]).all() and np.array_equal(v[0], x[0]) and np.array_equal(v[1, :32], x[1, :32])


def test_swiglu_gradients_by_differences():
    rng = _rng(3)
    g, u, dh = rng.normal(size=200) * 4, rng.normal(size=200), rng.normal(size=200)
    dg, du = R.swiglu_grad(dh, g, u)
    h = 1e-5
    # the central difference is off by h^2/6 of a third derivative (below 1 here times |dh u|) and rounding
    tol = (h * h + 4e-16 * (1 + np.abs(g)) / h) * (1 + np.abs(dh)) * (1 + np.abs(u))
    assert (np.abs(dg - dh * (R.swiglu(g + h, u) - R.swiglu(g - h, u)) / (2 * h)) <= tol).all()
    assert (np.abs(du - dh * (R.swiglu(g, u + h) - R.swiglu(g, u - h)) / (2 * h)) <= tol).all()


def test_wgrad_by_differences():
    rng = _rng(4)
    x, W, dy = rng.normal(size=(7, 5)), rng.normal(size=(3, 5)), rng.normal(size=(7, 3))
    G = R.wgrad(dy, x)
    for i in range(3):
        for j in range(5):
            E = np.zeros_like(W)
            E[i, j] = 0.5
            # linear in W: the difference is exact up to rounding
            d = (dy * (x @ (W + E).T - x @ (W - E).T)).sum()
            assert abs(G[i, j] - d) < 1e-13 * 35


def test_embedding_gradient_by_differences():
    rng = _rng(5)
    E, ids, dy = rng.normal(size=(6, 4)), np.array([1, 5, 1, 0, 3, 1, -1, 9]), rng.normal(size=(8, 4))
    G = R.embed_grad(dy, ids, 6, scale=2.5, pad_id=3)
    for v in range(6):
        for j in range(4):
            D = np.zeros_like(E)
            D[v, j] = 0.5
            d = (dy * (R.embed(E + D, ids, 2.5, 3) - R.embed(E - D, ids, 2.5, 3))).sum()
            assert abs(G[v, j] - d) < 1e-13 * 32
    assert not G[[2, 3, 4]].any()
