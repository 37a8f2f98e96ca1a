"""Values of the training-step operators where the arithmetic is at its limits,
against binary64."""
import numpy as np
import pytest
import torch

import paper_2607_19331_gb300 as iso
from oracle import train_step as R
from paper_2607_19331_gb300 import _abi

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24
ROUND = {BF: 2.0 ** -8, F32: U}          # half an ulp, relative
LEAST = {BF: 2.0 ** -133, F32: 2.0 ** -149}


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    torch.cuda.set_device(0)
    _abi.lib()


def _np(t):
    return t.detach().double().cpu().numpy()


def _within(got, ref, tol, what):
    d = np.abs(_np(got) - ref)
    assert (d <= tol).all(), f"{what}: worst {np.max(d / tol):.3g} of the bound"


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("up", [1.0, -3.0, 2.0 ** 60])
def test_swiglu_keeps_the_small_end_of_silu(dtype, up):
    """Gates where exp(-gate) nears binary32's largest number and passes it.
    Relative: the exponential's error (2 + 1.2 |gate| ulp where it is the fast
    one), a few roundings and the output's; absolute: two steps of a subnormal
    exp(-|gate|) times the factors, and one of the output."""
    g = torch.linspace(-92, -80, 97).reshape(1, 97).to(DEV, dtype)
    u = torch.full_like(g, up)
    h, gp, up_p = iso.swiglu_pack(g, u)
    dh = torch.ones_like(g)
    dg, du, hh = iso.swiglu_grad(dh, gp, up_p)

    def tol(ref, gate, factor):
        rel = ROUND[dtype] + (1 + ROUND[dtype]) * (16 + (2.5 * np.abs(gate) if dtype == BF else 0)) * U
        return rel * np.abs(ref) + 2 * 2.0 ** -149 * (1 + np.abs(gate)) * factor + LEAST[dtype]
    gv, uv = _np(g), _np(u)
    ref = R.swiglu(gv, uv)
    _within(h, ref, tol(ref, gv, abs(up)), "h")
    gv, uv = R.act_values(gv), R.act_values(uv)
    _within(hh, R.swiglu(gv, uv), tol(R.swiglu(gv, uv), gv, abs(up)), "h again")
    rg, ru = R.swiglu_grad(1.0, gv, uv)
    _within(du, ru, tol(ru, gv, 1.0), "d_up")
    # s (1 + g (1 - s)): the terms are s and |g| s
    _within(dg, rg, tol(np.abs(uv) * R.sigmoid(gv) * (1 + np.abs(gv)), gv, abs(up)), "d_gate")


# ---------------------------------------------------------------------------
# weight gradient: operands whose errors do not average out
# ---------------------------------------------------------------------------
def _wgrad_bound(T, dtype, mag, x_mag):
    """Inside the bound of include/iso.h: sixteen products at a time, each cut
    below 2^-25 of the largest term, the running sum below 2^-23 of itself;
    chains rounded."""
    P = T if dtype == BF else 3 * T
    return (min(P, 1024) * 5 * 2.0 ** -27 + (P / 1024 + 2) * U) * mag + (2.0 ** -133 * x_mag if dtype == F32 else 0)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [9, 100, 1024, 3000, 8192])
@pytest.mark.parametrize("kind", ["one sign", 2.0 ** -20, 2.0 ** -25, 2.0 ** -26, 2.0 ** -30, "rising"])
def test_wgrad_of_operands_of_one_sign(kind, T, dtype):
    M, N, g = 264, 160, torch.Generator().manual_seed(1)
    x = torch.ones(T, N)
    if kind == "one sign":
        dy, x = 0.5 + torch.rand(T, M, generator=g), 0.5 + torch.rand(T, N, generator=g)
    elif kind == "rising":
        dy = torch.exp2(torch.linspace(-30, 0, T))[:, None].expand(T, M).clone()
    else:                                     # one large product, then small ones
        dy = torch.full((T, M), kind)
        dy[0] = 1.0
    dy, p = dy.to(DEV, dtype), iso.act_pack(x.to(DEV, BF))
    xh, d = _np(iso.act_unpack(p)), _np(dy)
    ref = d.T @ xh
    got = iso.act_wgrad(dy, p)
    _within(got, ref, _wgrad_bound(T, dtype, d.T @ xh, xh.sum(0)) + U * ref, f"{kind}")
    _within(iso.act_wgrad(-dy, p), -ref, _wgrad_bound(T, dtype, d.T @ xh, xh.sum(0)) + U * ref, f"-{kind}")


@pytest.mark.parametrize("size", [2.0 ** -105, 2.0 ** -112, 2.0 ** -125, 2.0 ** -140])
@pytest.mark.parametrize("T", [9, 40, 2000])
def test_wgrad_of_tiny_gradients(T, size):
    """A binary32 dY near and below the least normal number."""
    g = torch.Generator().manual_seed(2)
    dy = (torch.randn(T, 270, generator=g) * size).to(DEV)
    p = iso.act_pack((torch.randn(T, 150, generator=g) * 2.0 ** 30).to(DEV))
    xh, d = _np(iso.act_unpack(p, dtype=F32)), _np(dy)
    mag, x_mag = np.abs(d).T @ np.abs(xh), np.abs(xh).sum(0)
    ref = d.T @ xh
    _within(iso.act_wgrad(dy, p), ref, _wgrad_bound(T, F32, mag, x_mag) + U * np.abs(ref) + 2.0 ** -149, f"{size}")
