"""Host-side checks of the operators between the embedding and the loss (no GPU
needed): the refusals that come before anything reaches the device."""
import ctypes
import math

import pytest
import torch

import paper_2607_19331_gb300 as iso
from paper_2607_19331_gb300 import _abi, decoder
from paper_2607_19331_gb300._abi import IsoAttnCfg, IsoMat, IsoRopeCfg

A = 0x100000000
WS = ctypes.c_void_p(0x40000000)
BIG = 1 << 40
BF, F32 = _abi.ISO_BF16, _abi.ISO_F32
ARG, SHAPE, DTYPE, ALIGN = _abi.ISO_ERR_ARG, _abi.ISO_ERR_SHAPE, _abi.ISO_ERR_DTYPE, _abi.ISO_ERR_ALIGN
UNSUPPORTED, WORKSPACE = _abi.ISO_ERR_UNSUPPORTED, _abi.ISO_ERR_WORKSPACE


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_19331_gb300 import build
    build.build()


def mat(rows, cols, ptr=A, ld=None, dtype=BF):
    return IsoMat(ptr, rows, cols, cols if ld is None else ld, dtype, 0)


def at(x):
    return ctypes.c_void_p(x)


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------
def rope(x, y, positions=9 * A, i64=1, ld=4, **change):
    freq, axis = (ctypes.c_double * 8)(*[1.0] * 8), (ctypes.c_int32 * 8)(*[0] * 8)
    for i, f in change.pop("freqs", {}).items():
        freq[i] = f
    for i, a in change.pop("axis_of", {}).items():
        axis[i] = a
    cfg = IsoRopeCfg(32, 16, 1, 0, 0, 0, ctypes.addressof(freq), ctypes.addressof(axis))
    for name, value in change.items():
        setattr(cfg, name, value)
    return _abi.lib().iso_rope(x, at(positions), i64, ld, cfg, y, None)


def test_rope_refusals():
    x, y = mat(4, 64), mat(4, 64, 2 * A)
    for bad in (dict(head_dim=0), dict(rot_dim=15), dict(rot_dim=34), dict(rot_dim=-2), dict(axes=0), dict(axes=5),
                dict(neighbours=2), dict(inverse=-1), dict(reserved=1), dict(freq=None), dict(axis=None),
                dict(freqs={3: math.inf}), dict(freqs={0: math.nan}), dict(axis_of={7: 1}), dict(axis_of={1: -1}), dict(i64=2)):
        assert rope(x, y, **bad) == ARG, bad
    assert rope(mat(4, 600, ld=600), mat(4, 600, 2 * A), head_dim=600, rot_dim=258) == ARG
    assert rope(mat(4, 65), mat(4, 65, 2 * A)) == SHAPE
    assert rope(x, mat(5, 64, 2 * A)) == SHAPE and rope(x, mat(4, 32, 2 * A)) == SHAPE
    assert rope(x, y, ld=3) == SHAPE and rope(x, y, ld=1 << 40) == UNSUPPORTED
    assert rope(x, mat(4, 64, 2 * A, dtype=F32)) == DTYPE and rope(mat(4, 64, dtype=7), y) == DTYPE
    assert rope(x, y, positions=9 * A + 4) == ALIGN and rope(x, y, positions=9 * A + 2, i64=0) == ALIGN
    assert rope(x, y, positions=0) == ARG
    assert rope(x, mat(4, 64, A + 2)) == ARG                         # over x, not x
    assert rope(x, mat(4, 64, ld=66)) == ARG
    assert rope(x, y, positions=2 * A + 64) == ARG                   # the output over the positions
    assert rope(mat(0, 64, None), mat(0, 64, None), positions=0) == _abi.ISO_OK
    assert rope(mat(4, 0, None), mat(4, 0, None), positions=0) == _abi.ISO_OK


def test_rope_plans():
    p = iso.rope_plan(128, base=1e6, sections=(16, 24, 24))
    assert (p.rot_dim, p.axes) == (128, 3) and list(p.axis) == [0] * 16 + [1] * 24 + [2] * 24
    assert list(p.freq) == [1e6 ** (-i / 64) for i in range(64)]
    p = iso.rope_plan(64, rot_dim=16, sections=(4, 2, 2), turns=True, per_axis=True)
    assert list(p.axis) == [0, 1, 2, 0, 1, 2, 0, 0]
    assert list(p.freq) == [1.0, 1.0, 1.0, 1e4 ** -0.25, 1e4 ** -0.5, 1e4 ** -0.5, 1e4 ** -0.5, 1e4 ** -0.75]
    assert iso.rope_plan(6, rot_dim=0).rot_dim == 0
    for bad in (dict(rot_dim=7), dict(rot_dim=130), dict(base=0.0), dict(sections=(1, 2)), dict(sections=(65, -1)),
                dict(sections=()), dict(sections=(60, 1, 1, 1, 1)), dict(pairs="other")):
        with pytest.raises(ValueError):
            iso.rope_plan(128, **bad)
    with pytest.raises(ValueError):
        iso.rope_plan(300)
    with pytest.raises(ValueError):
        iso.RopePlan(8, [1.0, math.inf], [0, 0], 1)
    with pytest.raises(ValueError):
        iso.RopePlan(8, [1.0], [0, 0], 1)


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def cfg(heads=4, kv=2, dim=64, causal=1, window=0, scale=0.125, n=0, q_ends=None, k_ends=None, rest=0, reserved=0):
    return IsoAttnCfg(heads, kv, dim, causal, window, scale, n, q_ends, k_ends, rest, reserved)


def attn(q=None, k=None, v=None, out=None, c=None, lse=5 * A, ws=WS, n=BIG, status=None):
    return _abi.lib().iso_attn(q or mat(10, 256), k or mat(10, 128, 2 * A), v or mat(10, 128, 3 * A), c or cfg(),
                               out or mat(10, 256, 4 * A), at(lse), ws, n, status, None)


def test_attention_refusals():
    for bad in (cfg(heads=0), cfg(kv=0), cfg(kv=3), cfg(dim=0), cfg(causal=2), cfg(window=-1), cfg(window=4, causal=0),
                cfg(scale=0.0), cfg(scale=-1.0), cfg(scale=math.nan), cfg(scale=math.inf), cfg(n=-1), cfg(n=2),
                cfg(q_ends=6 * A), cfg(k_ends=6 * A), cfg(rest=2), cfg(reserved=1)):
        assert attn(c=bad) == ARG
    assert attn(c=cfg(n=1, q_ends=6 * A + 2)) == ALIGN
    assert attn(c=cfg(dim=129)) == UNSUPPORTED
    assert attn(q=mat(10, 255)) == SHAPE and attn(k=mat(10, 256, 2 * A)) == SHAPE and attn(v=mat(9, 128, 3 * A)) == SHAPE
    assert attn(out=mat(9, 256, 4 * A)) == SHAPE
    assert attn(k=mat(9, 128, 2 * A), v=mat(9, 128, 3 * A), c=cfg(n=1, q_ends=6 * A)) == SHAPE      # no offsets of the keys'
    assert attn(q=mat((1 << 30) + 1, 256), out=mat((1 << 30) + 1, 256, 4096 * A)) == UNSUPPORTED
    assert attn(k=mat(10, 128, 2 * A, dtype=F32)) == DTYPE and attn(v=mat(10, 128, 3 * A, dtype=F32)) == DTYPE
    assert attn(out=mat(10, 256, 4 * A, dtype=F32)) == DTYPE
    assert attn(lse=0) == ARG and attn(lse=5 * A + 2) == ALIGN
    assert attn(out=mat(10, 256, A + 2)) == ARG and attn(out=mat(10, 256, 2 * A)) == ARG            # over an input
    assert attn(lse=4 * A) == ARG and attn(lse=3 * A + 64) == ARG                                   # lse over out, over v
    assert attn(c=cfg(n=1, q_ends=4 * A)) == ARG                                                    # out over the offsets
    assert attn(ws=None) == WORKSPACE and attn(n=16) == WORKSPACE and attn(ws=ctypes.c_void_p(0x40000010)) == WORKSPACE
    nb = ctypes.c_size_t()
    assert _abi.lib().iso_attn_workspace_size(mat(10, 256), mat(10, 128), cfg(), None) == ARG
    assert _abi.lib().iso_attn_workspace_size(mat(10, 256), mat(10, 64), cfg(), nb) == SHAPE
    empty = mat(0, 256, None)
    assert attn(q=empty, out=empty, lse=0) == _abi.ISO_OK                                           # no queries


def grad(c=None, ws=WS, n=BIG, **m):
    d = dict(dout=mat(10, 256, 7 * A), q=mat(10, 256), k=mat(10, 128, 2 * A), v=mat(10, 128, 3 * A), out=mat(10, 256, 4 * A),
             dq=mat(10, 256, 8 * A), dk=mat(10, 128, 9 * A), dv=mat(10, 128, 10 * A), lse=5 * A)
    d.update(m)
    return _abi.lib().iso_attn_grad(d["dout"], d["q"], d["k"], d["v"], d["out"], at(d["lse"]), c or cfg(), d["dq"], d["dk"],
                                    d["dv"], ws, n, None, None)


def test_attention_gradient_refusals():
    assert grad(c=cfg(kv=3)) == ARG and grad(c=cfg(dim=130)) == UNSUPPORTED
    for name, shape in dict(dout=(10, 255), out=(9, 256), dq=(10, 128), dk=(10, 256), dv=(11, 128), v=(10, 64)).items():
        assert grad(**{name: mat(*shape, 20 * A)}) == SHAPE, name
    for name, shape in dict(dout=(10, 256), out=(10, 256), dq=(10, 256), dk=(10, 128), dv=(10, 128), k=(10, 128)).items():
        assert grad(**{name: mat(*shape, 20 * A, dtype=F32)}) == DTYPE, name
    assert grad(lse=0) == ARG and grad(lse=5 * A + 1) == ALIGN
    assert grad(dq=mat(10, 256, A)) == ARG and grad(dk=mat(10, 128, 9 * A), dv=mat(10, 128, 9 * A + 64)) == ARG
    assert grad(dv=mat(10, 128, 5 * A)) == ARG and grad(dq=mat(10, 256, 7 * A)) == ARG
    nb = ctypes.c_size_t()
    L = _abi.lib()
    assert L.iso_attn_grad_workspace_size(mat(10, 256), mat(10, 128), cfg(), nb) == 0 and nb.value >= 4 * 10 * 4
    assert grad(n=nb.value - 1) == WORKSPACE and grad(ws=None) == WORKSPACE
    # ranges of one buffer pass the check of overlap (the refusal is the workspace's)
    parts = dict(dq=mat(10, 256, 8 * A, ld=512), dk=mat(10, 128, 8 * A + 512, ld=512), dv=mat(10, 128, 8 * A + 768, ld=512))
    assert grad(ws=None, **parts) == WORKSPACE


# ---------------------------------------------------------------------------
# distillation
# ---------------------------------------------------------------------------
def distill(z=None, ids=2 * A, i64=1, t=None, tau=1.0, loss=4 * A, lse=5 * A, dloss=6 * A, g=None):
    return _abi.lib().iso_distill(z or mat(10, 100), at(ids), i64, t or mat(10, 8, 3 * A), tau, at(loss), at(lse), at(dloss),
                                  g, None, None)


def distill_grad(z=None, ids=2 * A, t=None, tau=1.0, lse=5 * A, dloss=6 * A, g=None):
    return _abi.lib().iso_distill_grad(at(dloss), z or mat(10, 100), at(ids), 1, t or mat(10, 8, 3 * A), tau, at(lse),
                                       g, None, None)


def test_distillation_refusals():
    out = mat(10, 100, 8 * A)
    for tau in (0.0, -1.0, math.inf, math.nan, 1e-45):
        assert distill(tau=tau) == ARG and distill_grad(tau=tau, g=out) == ARG
    assert distill(i64=2) == ARG and distill(ids=0) == ARG and distill(loss=0) == ARG and distill(lse=0) == ARG
    assert distill(g=out, dloss=0) == ARG and distill_grad(g=None) == ARG and distill_grad(g=out, lse=0) == ARG
    assert distill(ids=2 * A + 4) == ALIGN and distill(loss=4 * A + 1) == ALIGN and distill_grad(g=out, dloss=6 * A + 2) == ALIGN
    assert distill(t=mat(9, 8, 3 * A)) == SHAPE and distill(g=mat(10, 99, 8 * A)) == SHAPE
    assert distill(t=mat(10, 2049, 3 * A)) == UNSUPPORTED
    assert distill(g=mat(10, 100, 8 * A, dtype=F32)) == DTYPE and distill(t=mat(10, 8, 3 * A, dtype=9)) == DTYPE
    assert distill(g=mat(10, 100, A + 2)) == ARG and distill(g=mat(10, 100, A, ld=101)) == ARG      # over the logits, not them
    assert distill(g=mat(10, 100, 3 * A)) == ARG and distill(g=mat(10, 100, 2 * A)) == ARG
    assert distill(loss=5 * A, lse=5 * A) == ARG and distill(loss=A) == ARG and distill(g=out, loss=8 * A) == ARG
    assert distill_grad(g=mat(10, 100, 5 * A)) == ARG and distill_grad(g=mat(10, 100, 6 * A)) == ARG
    none = mat(0, 100, None)
    assert distill(z=none, t=mat(0, 8, None), ids=0, loss=0, lse=0, dloss=0) == _abi.ISO_OK


# ---------------------------------------------------------------------------
# the binding
# ---------------------------------------------------------------------------
def test_python_checks_without_a_gpu():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    plan = iso.rope_plan(32)
    with pytest.raises(TypeError, match="RopePlan"):
        iso.rope(x, torch.zeros(4, dtype=torch.int64), None)
    with pytest.raises(TypeError, match="RopePlan"):
        iso.rope_grad(x, torch.zeros(4, dtype=torch.int64), "plan")
    with pytest.raises(ValueError, match="CUDA"):
        iso.rope(x, torch.zeros(4, dtype=torch.int64), plan)
    with pytest.raises(ValueError, match="CUDA"):
        iso.attn(x, x, x, 2)
    with pytest.raises(TypeError, match="bfloat16 or float32"):
        iso.attn(x.half(), x, x, 2)
    with pytest.raises(ValueError, match="CUDA"):
        iso.distill(x, torch.zeros(4, 2, dtype=torch.int64), x)
    q = mat(4, 64)

    def of(heads=2, kv=None, scale=None, causal=True, window=0, seqs=None, kv_seqs=None):
        return decoder._attn_cfg(q, heads, kv, scale, causal, window, seqs, kv_seqs)
    for bad in (dict(heads=0), dict(heads=3), dict(kv=3), dict(kv=0), dict(window=-1), dict(window=3, causal=False),
                dict(scale=0.0), dict(scale=math.nan)):
        with pytest.raises(ValueError):
            of(**bad)
    for seqs in (torch.zeros(3), torch.zeros(1, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)):
        with pytest.raises(TypeError, match="offsets"):
            of(seqs=seqs)
    c = of(heads=4, kv=2)
    assert (c.heads, c.kv_heads, c.head_dim, c.scale, c.n_seqs) == (4, 2, 16, 0.25, 0)
    for tau in (0, -1, math.inf, math.nan):
        with pytest.raises(ValueError):
            decoder._tau(tau)
