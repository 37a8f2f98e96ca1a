"""Distillation of finite logits of any size: vocabularies masked by the type's lowest value
or by -1e10, whole rows of such numbers, against oracle/decoder_step.py in binary64.

Loss and gradient do not change when a row is shifted, so the oracle takes rows less
their maximum, Z, with what lies 1e6 tau below it at -Inf (its weight is 0 in binary64
too).  Bounds (U = 2^-24, fast = 2^-21 for bfloat16, as in test_gpu_decoder.py): a score
(x - m) / tau is off by 3 U |Z| / tau, a sum of V exponentials by n = (V / 128 + 64) U + fast
relative; log s by that and U |log s|; lse by 3 U |m| / tau more; a probability by all
three; from lse by U |lse| more, and E = eps / 2 of the gradient's type for its rounding."""
import math

import numpy as np
import pytest
import torch

import paper_2607_19331_gb300 as iso
from oracle import decoder_step as R
from paper_2607_19331_gb300 import _abi

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
E = {BF: 2.0 ** -8, F32: U}


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    torch.cuda.set_device(0)
    _abi.lib()


def _np(t):
    return t.detach().double().cpu().numpy()


# kinds of rows, the others are ordinary; the teacher's ids are KEPT entries in all but TO_MASKED
KEPT, TO_MASKED, WHOLE, TWO, FEW, PART, BLOCKS = 5, 0, 1, 2, 3, 4, 5


def _case(T, V, K, dtype, low):
    g = torch.Generator(DEV).manual_seed(T + V)
    z = (torch.randn(T, V, generator=g, device=DEV) * 3).to(dtype)
    ids = torch.randint(0, KEPT, (T, K), generator=g, device=DEV)
    ids = torch.tensor([V // 3, V // 3 + 1, V // 2, V - 2, 1], device=DEV)[ids]
    keep = torch.zeros(V, dtype=torch.bool, device=DEV)
    keep[ids.unique()] = True
    block = (torch.arange(V, device=DEV) // max(1, V // 16)) % 2 == 0
    z[FEW] = torch.where(keep, z[FEW], low)
    z[PART] = torch.where(keep | (torch.arange(V, device=DEV) > V // 4), z[PART], low)
    z[BLOCKS] = torch.where(keep | block, z[BLOCKS], low)
    z[TO_MASKED] = z[BLOCKS]
    ids[TO_MASKED] = int((~(keep | block)).nonzero()[0])
    z[WHOLE] = low
    z[TWO] = low
    z[TWO, [1, V // 2]] = low / 2
    ids[TWO] = torch.where(ids[TWO] == 1, 1, V // 2)
    t, d = torch.randn(T, K, generator=g, device=DEV), torch.randn(T, generator=g, device=DEV)
    return z, ids, t.to(dtype), d


def _check(z, ids, t, d, tau, loss, lse, grad, what, from_lse=False):
    """Rows of one call; loss or grad may be None."""
    dtype, V, K = z.dtype, z.shape[1], ids.shape[1]
    z, ids, t, d = _np(z), ids.cpu().numpy(), _np(t), _np(d)
    top = z.max(1, keepdims=True)
    Z = z - top
    Z[Z < -1e6 * tau] = -np.inf
    want_loss, s, want = R.distill(Z, ids, t, tau, d)
    fast = 2.0 ** -21 if dtype == BF else 0.0
    size = np.abs(np.where(np.isfinite(Z), Z, 0)) / tau
    far = 3 * U * size.max(1) + (V / 128 + 64) * U + fast + 2 * U * np.abs(s)          # of log s
    m = np.abs(top[:, 0]) / tau
    if loss is not None:
        e = tau ** 2 * (far + 8 * U * (np.abs(t).max(1) / tau + size.max(1) + np.abs(s) + 8 + K)) + 4 * U * np.abs(want_loss)
        assert (np.abs(_np(loss) - want_loss) <= e).all(), (what, "loss", _np(loss), want_loss)
        with np.errstate(over="ignore"):
            assert (np.abs(_np(lse) - (s + top[:, 0] / tau)) <= far + 4 * U * (m + np.abs(s))).all(), (what, "lse")
    q = np.exp(Z / tau - s[:, None])
    other = np.abs(want / (d * tau)[:, None] - q)
    off = far + (U * (4 * m + np.abs(s)) if from_lse else 0)
    e = np.abs(d * tau)[:, None] * (q * (3 * U * size + off[:, None] + 8 * U + fast) + U * 16 * (2 + K / 8) * (other + q))
    got = _np(grad)
    ok = np.abs(got - want) <= e + E[dtype] * np.abs(want) + 1e-36
    assert ok.all(), (what, "gradient", [(int(r), int(c), got[r, c], want[r, c]) for r, c in np.argwhere(~ok)[:4]])


# a CTA's registers, a cluster's, streamed by one CTA and by several, entry by entry
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("mask,tau", [("lowest", 1.0), ("lowest", 0.7), ("lowest", 2.0), (-1e10, 1.0)])
@pytest.mark.parametrize("T,V,K,aside", [
    (8, 60, 3, False), (8, 3000, 9, False), (8, 9001, 20, False), (8, 60001, 300, False), (8, 152064, 64, False),
    (700, 32000, 20, False), (700, 16000, 20, False), (2600, 60000, 8, False), (8, 3000, 9, True), (8, 60001, 20, True)])
def test_finite_masks(T, V, K, aside, mask, tau, dtype):
    low = torch.finfo(dtype).min if mask == "lowest" else mask
    z, ids, t, d = _case(T, V, K, dtype, low)
    if aside:
        buf = torch.empty(T, V + 3, dtype=dtype, device=DEV)
        loss, lse, grad = iso.distill(z, ids, t, tau, dloss=d, out=buf[:, 3:])
    else:
        loss, lse, grad = iso.distill(z, ids, t, tau, dloss=d)
    l2, s2 = iso.distill(z, ids, t, tau)
    apart = iso.distill_grad(d, z, ids, t, lse, tau)
    overflow = mask == "lowest" and tau < 1                    # lse of the whole row is beyond binary32
    assert torch.isinf(lse).sum() == overflow and torch.isinf(s2).sum() == overflow and not torch.isnan(lse).any()
    part = [WHOLE, TWO, FEW, PART, BLOCKS, 6, T - 1]
    pick = lambda x: x[part]                                   # noqa: E731
    # lse of such rows is as near as binary32 is there; loss and gradient do not hang on it
    same = lambda s: torch.where(torch.isinf(s), pick(z).double().amax(1) / tau, s.double()) if overflow else s     # noqa: E731
    _check(pick(z), pick(ids), pick(t), pick(d), tau, pick(loss), same(pick(lse)), pick(grad), "joint")
    _check(pick(z), pick(ids), pick(t), pick(d), tau, pick(l2), same(pick(s2)), pick(grad), "loss alone")
    ordinary = [FEW, PART, BLOCKS, 6, T - 1]
    _check(z[ordinary], ids[ordinary], t[ordinary], d[ordinary], tau, None, None, apart[ordinary], "apart", from_lse=True)
    assert torch.isfinite(apart).all()
    # a masked entry has no weight and the teacher's whole: its gradient is -dloss tau, its loss tau (m - low)
    want = tau * (_np(z[TO_MASKED]).max() - float(torch.tensor(low, dtype=dtype)))
    for got in (loss, l2):
        assert abs(float(got[TO_MASKED].double()) - want) <= 64 * U * want or want / min(tau, 1) > 3.402e38 and math.isinf(got[TO_MASKED])
    id0 = int(ids[TO_MASKED, 0])
    for got in (grad, apart):
        assert abs(float(got[TO_MASKED, id0]) / float(-d[TO_MASKED] * tau) - 1) <= (K + 16) * U + E[dtype]
    # rows that a program does not train on stay 0
    for got in (iso.distill(z, ids, t, tau, dloss=torch.zeros_like(d))[2], iso.distill_grad(torch.zeros_like(d), z, ids, t, lse, tau)):
        assert (got == 0).all()


@pytest.mark.parametrize("low", ["lowest", -1e10])
def test_a_teachers_masks(low):
    """Its used slots, all of them at the lowest value: a distribution like any other."""
    for dtype in (BF, F32):
        v = torch.finfo(dtype).min if low == "lowest" else low
        z, ids, _, d = _case(8, 3000, 4, dtype, -3.0)
        t = torch.full((8, 4), v, dtype=dtype, device=DEV)
        t[5, 1] = 0.5
        for tau in (0.7, 1.0, 2.0):
            loss, lse, grad = iso.distill(z, ids, t, tau, dloss=d)
            flat = torch.zeros(8, 4, dtype=dtype, device=DEV)
            flat[5], flat[5, 1] = -math.inf, 0.0
            want = iso.distill(z, ids, flat, tau, dloss=d)
            assert all(torch.equal(a, b) for a, b in zip((loss, lse, grad), want))
