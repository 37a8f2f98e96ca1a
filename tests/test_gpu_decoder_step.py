"""The operators between the embedding and the loss together, as
examples/decoder_step.py uses them: the gradients of a whole step against the
same chain in binary64."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import decoder_step as D
from oracle import train_step as R

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    torch.cuda.set_device(0)
    spec = importlib.util.spec_from_file_location("decoder_step", os.path.join(ROOT, "examples", "decoder_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _np(t):
    return t.detach().double().cpu().numpy()


def test_step_gradients_match_binary64(example):
    """Every stage is binary32 with sums of at most 400 terms, so it adds an error of
    at most (400 + 16) 2^-24 = 2.5e-5 of the norm of its terms' magnitudes; sums of
    random signs cancel to about a twentieth of those (n^-1/2), and twelve stages
    follow one another: 12 * 2.5e-5 * 20 = 6e-3 at the very worst, and errors of
    random sign stay below a hundredth of it.  1e-4 of the gradient's norm is held."""
    V, H, KV, dim, lengths, pad = 300, 4, 2, 32, [37, 1, 29], 4
    torch.backends.cuda.matmul.allow_tf32 = False
    ids, positions, seqs, top_ids, top_logits, weights = example.batch(V, lengths, pad, 8)
    model = example.Block(V, H, KV, dim, dtype=torch.float32, seed=3, pad_id=V - 1)
    logits, kept = model.forward(ids, positions, seqs)
    loss, lse, dlogits = example.iso.distill(logits, top_ids, top_logits, dloss=weights)
    g_E, g_qkv, g_out = model.backward(ids, positions, seqs, dlogits, kept)

    E, Wz, Wo, i = _np(model.E), _np(model.qkv), _np(model.out), ids.cpu().numpy()
    x = R.embed(E, i, model.scale, V - 1)
    freq, axis, pos = list(model.plan.freq), list(model.plan.axis), positions.cpu().numpy()[None]
    z = x @ Wz.T
    n = (H + KV) * dim
    z[:, :n] = D.rope(z[:, :n], pos, dim, freq, axis)
    T = len(x)
    o, l = np.zeros((T, H * dim)), np.zeros((H, T))

    def parts():
        at = 0
        for m in lengths:
            for h in range(H):
                g = h // (H // KV)
                yield (h, slice(at, at + m), slice(h * dim, (h + 1) * dim), slice((H + g) * dim, (H + g + 1) * dim),
                       slice((H + KV + g) * dim, (H + KV + g + 1) * dim), D.sees(m, m, True, 0))
            at += m
    for h, rows, qc, kc, vc, seen in parts():
        o[rows, qc], l[h, rows], _ = D.attn(z[rows, qc], z[rows, kc], z[rows, vc], dim ** -0.5, seen)
    y = x + o @ Wo.T
    ref_logits = y @ E.T
    ref_loss, _, ref_d = D.distill(ref_logits, top_ids.cpu().numpy(), _np(top_logits), 1.0, _np(weights))

    def near(got, ref, what):
        got = _np(got) if isinstance(got, torch.Tensor) else got
        err = np.linalg.norm(got - ref) / np.linalg.norm(ref)
        assert err <= 1e-4, f"{what}: {err:.2e}"
    near(logits, ref_logits, "logits")
    near(loss, ref_loss, "loss")
    near(dlogits, ref_d, "dlogits")
    dy = ref_d @ E
    do = dy @ Wo
    dz = np.zeros_like(z)
    for h, rows, qc, kc, vc, seen in parts():
        a, b, c = D.attn_grad(do[rows, qc], z[rows, qc], z[rows, kc], z[rows, vc], o[rows, qc], l[h, rows], dim ** -0.5, seen)
        dz[rows, qc] += a
        dz[rows, kc] += b
        dz[rows, vc] += c
    dz[:, :n] = D.rope(dz[:, :n], pos, dim, freq, axis, inverse=True)
    # the weight gradients take the checkpoints' values, which are the same on both sides
    # but where a rounding apart moves one by a step of its group (a 127th of its largest)
    unpack = lambda p: _np(example.iso.act_unpack(p, dtype=torch.float32))                     # noqa: E731
    near(g_qkv, R.wgrad(dz, unpack(kept[0])), "q-k-v projection")
    near(g_out, R.wgrad(dy, unpack(example.iso.act_pack(kept[2]))), "output projection")
    dx = dy + dz @ Wz
    near(g_E, R.wgrad(ref_d, unpack(example.iso.act_pack(kept[4]))) + R.embed_grad(dx, i, V, model.scale, V - 1), "table")


def test_the_example_runs(example):
    losses = example.main(steps=2)
    assert len(losses) == 2 and all(np.isfinite(losses))
