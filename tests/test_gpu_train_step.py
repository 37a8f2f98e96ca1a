"""The training-step operators together, as examples/mlp_step.py uses them: the
gradients of a whole step against the same chain in binary64, and a few steps
under ISO[AdamW]."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import train_step as R

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    torch.cuda.set_device(0)
    spec = importlib.util.spec_from_file_location("mlp_step", os.path.join(ROOT, "examples", "mlp_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _np(t):
    return t.detach().double().cpu().numpy()


def test_step_gradients_match_binary64(example):
    V, H, INTER, T = 200, 96, 160, 70
    model = example.Block(V, H, INTER, dtype=torch.float32, seed=3, pad_id=V - 1)
    gen = torch.Generator(device="cuda").manual_seed(5)
    ids = torch.randint(0, V, (T,), generator=gen, device="cuda")
    dy = torch.randn(T, H, generator=gen, device="cuda") * 1e-2
    torch.backends.cuda.matmul.allow_tf32 = False
    y, kept = model.forward(ids)
    g_E, g_gu, g_down = model.backward(ids, dy, kept)

    E, Wgu, Wd, i, d = _np(model.E), _np(model.gate_up.W), _np(model.down.W), ids.cpu().numpy(), _np(dy)
    x = R.embed(E, i, model.scale, V - 1)
    z = x @ Wgu.T
    ref_y = R.swiglu(z[:, :INTER], z[:, INTER:]) @ Wd.T
    # every factor carries a binary32 rounding or a sum of n of them: n + 16 roundings of the sum of magnitudes
    U = 2.0 ** -24
    ax, aW = np.abs(x), np.abs(Wgu)
    tol_z = (H + 16) * U * (ax @ aW.T)
    mag_h = (np.abs(z) + tol_z)[:, :INTER] * (np.abs(z) + tol_z)[:, INTER:]
    assert (np.abs(_np(y) - ref_y) <= (2 * (H + INTER) + 64) * U * ((mag_h + ax.sum(1, keepdims=True) * aW.max()) @ np.abs(Wd).T) + 1e-30).all()

    # the backward pass from the checkpoints that were kept
    x_hat = _np(example.iso.act_unpack(kept[0], dtype=torch.float32))
    g, u = (_np(example.iso.act_unpack(p, dtype=torch.float32)) for p in kept[1:])
    assert (np.abs(x_hat - x) <= np.abs(x).max() / 127 + 1e-6).all()
    dh = d @ Wd
    dg, du = R.swiglu_grad(dh, g, u)
    dz = np.concatenate([dg, du], 1)
    mag_dh = np.abs(d) @ np.abs(Wd)
    s = R.sigmoid(g)
    tol_dh = (H + 4) * U * mag_dh
    tol_dz = np.concatenate([(tol_dh + 24 * U * np.abs(dh)) * np.abs(u) * s * (1 + np.abs(g)),
                             (tol_dh + 24 * U * np.abs(dh)) * np.abs(g) * s], 1) + 1e-30
    ref = dz.T @ x_hat
    tol = tol_dz.T @ np.abs(x_hat) + 4 * U * (8 + np.sqrt(T)) * (np.abs(dz).T @ np.abs(x_hat)) + U * np.abs(ref)
    assert (np.abs(_np(g_gu) - ref) <= tol).all()
    h = R.swiglu(g, u)
    h_hat = R.act_values(h.astype(np.float32))
    # h's own binary32 error can move a value across a rounding boundary of its checkpoint: one step of its group
    step = np.repeat(np.abs(np.pad(h, ((0, 0), (0, -INTER % 32)))).reshape(T, -1, 32).max(2) * 2 / 127, 32, axis=1)[:, :INTER]
    tol = np.abs(d).T @ (step * (np.abs(h_hat - h) > 0.49 * step)) + 4 * U * (8 + np.sqrt(T)) * (np.abs(d).T @ np.abs(h_hat))
    ref = d.T @ h_hat
    assert (np.abs(_np(g_down) - ref) <= tol + U * np.abs(ref) + np.abs(d).T @ (step * 0.02)).all()
    dx = dz @ Wgu
    tol_dx = tol_dz @ np.abs(Wgu) + (2 * INTER + 4) * U * (np.abs(dz) @ np.abs(Wgu))
    ref = R.embed_grad(dx, i, V, model.scale, V - 1)
    tol = R.embed_grad(tol_dx + (T + 4) * U * np.abs(dx), i, V, model.scale, V - 1)
    assert (np.abs(_np(g_E) - ref) <= tol + U * np.abs(ref)).all()
    assert not _np(g_E)[V - 1].any()


def test_a_step_changes_the_loss_as_its_gradients_say(example):
    """loss(after) - loss(before) against <gradients, changes> of one small step,
    the loss in binary64.  The gradients see activations off by at most 1/127 of
    their group's largest, half of it on average with random signs (about 1 % of
    a typical entry, far less in a sum of thousands); the step's second-order
    part is below lr times the curvature.  5 % covers both."""
    model = example.Block(300, 64, 128, dtype=torch.float32, seed=7)
    gen = torch.Generator(device="cuda").manual_seed(8)
    ids = torch.randint(0, 300, (256,), generator=gen, device="cuda")
    target = 0.1 * torch.randn(256, 64, generator=gen, device="cuda")

    def loss():
        E, Wgu, Wd = _np(model.E), _np(model.gate_up.W), _np(model.down.W)
        z = R.embed(E, ids.cpu().numpy(), model.scale) @ Wgu.T
        return np.square(R.swiglu(z[:, :128], z[:, 128:]) @ Wd.T - _np(target)).mean()
    y, kept = model.forward(ids)
    diff = y - target
    grads = [_np(g) for g in model.backward(ids, diff * (2.0 / diff.numel()), kept)]
    before, l0 = [_np(model.E), _np(model.gate_up.W), _np(model.down.W)], loss()
    s0 = torch.linalg.svdvals(model.down.W.double())
    model.step(ids, target, lr=1e-4, lr_embed=1e-2)
    after = [_np(model.E), _np(model.gate_up.W), _np(model.down.W)]
    change = sum((g * (b - a)).sum() for g, a, b in zip(grads, before, after))
    assert change < 0 and abs(loss() - l0 - change) <= 0.05 * abs(change)
    # the step's spectrum is exact up to the binary32 storage of W and its products
    s1 = torch.linalg.svdvals(model.down.W.double())
    assert (s1 - s0).abs().max() <= 1e-4 * s0.max()
