"""Host-side checks of the training-step entry points (no GPU needed): sizing
calls and the refusals that come before anything reaches the device."""
import ctypes

import pytest
import torch

import paper_2607_19331_gb300 as iso
from paper_2607_19331_gb300 import _abi
from paper_2607_19331_gb300._abi import IsoAct, IsoMat

A = 0x100000000
WS = ctypes.c_void_p(0x40000000)
BIG = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_19331_gb300 import build
    build.build()


def mat(rows, cols, ld=None, dtype=_abi.ISO_BF16, ptr=A, reserved=0):
    return IsoMat(ptr, rows, cols, cols if ld is None else ld, dtype, reserved)


def act(rows, cols, ptr=2 * A, eptr=3 * A, ldc=None, lde=None):
    groups = -(-cols // 32)
    return IsoAct(ptr, eptr, rows, cols, groups * 32 if ldc is None else ldc, -(-groups // 8) * 8 if lde is None else lde)


def test_new_status_has_a_text():
    assert _abi.lib().iso_error_string(_abi.ISO_ERR_INDEX).decode().startswith("ISO_ERR_INDEX")


def test_pack_refusals():
    L = _abi.lib()

    def pack(x, p):
        return L.iso_act_pack(x, p, None)
    assert pack(mat(4, 64), act(4, 96)) == _abi.ISO_ERR_SHAPE
    assert pack(mat(4, 64), act(5, 64)) == _abi.ISO_ERR_SHAPE
    assert pack(mat(4, 64, ld=63), act(4, 64)) == _abi.ISO_ERR_SHAPE
    assert pack(mat(-1, 64), act(-1, 64)) == _abi.ISO_ERR_SHAPE
    assert pack(mat(1 << 31, 64), act(1 << 31, 64)) == _abi.ISO_ERR_UNSUPPORTED
    assert pack(mat(4, 64, dtype=2), act(4, 64)) == _abi.ISO_ERR_DTYPE
    assert pack(mat(4, 64, reserved=1), act(4, 64)) == _abi.ISO_ERR_ARG
    assert pack(mat(4, 64, ptr=A + 1), act(4, 64)) == _abi.ISO_ERR_ALIGN
    assert pack(mat(4, 64, ptr=None), act(4, 64)) == _abi.ISO_ERR_ARG
    assert pack(mat(4, 64), act(4, 64, ptr=None)) == _abi.ISO_ERR_ARG
    assert pack(mat(4, 64), act(4, 64, ptr=2 * A + 8)) == _abi.ISO_ERR_ALIGN
    assert pack(mat(4, 64), act(4, 64, eptr=3 * A + 4)) == _abi.ISO_ERR_ALIGN
    assert pack(mat(4, 64), act(4, 64, ldc=65)) == _abi.ISO_ERR_ALIGN
    assert pack(mat(4, 64), act(4, 64, ldc=32)) == _abi.ISO_ERR_SHAPE
    assert pack(mat(4, 300), act(4, 300, lde=8)) == _abi.ISO_ERR_SHAPE
    assert pack(None, act(4, 64)) == _abi.ISO_ERR_ARG and pack(mat(4, 64), None) == _abi.ISO_ERR_ARG
    # codes over x, exponents over x, exponents over codes
    assert pack(mat(4, 64), act(4, 64, ptr=A + 256)) == _abi.ISO_ERR_ARG
    assert pack(mat(4, 64), act(4, 64, eptr=A + 504)) == _abi.ISO_ERR_ARG
    assert pack(mat(4, 64), act(4, 64, eptr=2 * A + 64)) == _abi.ISO_ERR_ARG
    # empty matrices need no data
    assert pack(mat(0, 64, ptr=None), act(0, 64, ptr=None, eptr=None)) == _abi.ISO_OK
    assert pack(mat(4, 0, ptr=None), act(4, 0, ptr=None, eptr=None)) == _abi.ISO_OK


def test_overlap_of_strided_matrices():
    """Through swiglu_grad's outputs on empty-of-launch refusals: halves of one
    buffer pass the overlap check, a shared column does not."""
    L = _abi.lib()
    bad_dtype = mat(4, 64, ptr=9 * A, dtype=_abi.ISO_F32)

    def grad(dg, du, dh=None):
        # dh of another dtype than h: a refusal either way, DTYPE before ARG only when shapes pass
        return L.iso_swiglu_grad(dh or mat(4, 64), act(4, 64), act(4, 64, ptr=4 * A, eptr=5 * A), dg, du, None, None)
    assert grad(bad_dtype, mat(4, 64, ptr=8 * A)) == _abi.ISO_ERR_DTYPE
    left, right = mat(4, 64, ld=128, ptr=8 * A), mat(4, 64, ld=128, ptr=8 * A + 126)
    assert grad(left, right) == _abi.ISO_ERR_ARG                      # one shared column
    assert grad(mat(4, 64, ptr=8 * A), mat(4, 64, ptr=8 * A + 2)) == _abi.ISO_ERR_ARG
    assert grad(mat(4, 64, ptr=A), mat(4, 64, ptr=8 * A)) == _abi.ISO_ERR_ARG       # over dh
    assert grad(mat(4, 64, ptr=2 * A), mat(4, 64, ptr=8 * A)) == _abi.ISO_ERR_ARG   # over a checkpoint
    assert grad(mat(4, 65), mat(4, 64, ptr=8 * A)) == _abi.ISO_ERR_SHAPE


def test_wgrad_sizes_and_refusals():
    L = _abi.lib()
    nb = ctypes.c_size_t()

    def size(dy, p, out):
        rc = L.iso_act_wgrad_workspace_size(dy, p, out, nb)
        return rc if rc else nb.value

    def run(dy, p, out, acc=0, ws=WS, n=BIG):
        return L.iso_act_wgrad(dy, p, out, acc, ws, n, None, None)
    out = mat(96, 64, ptr=6 * A)
    assert size(mat(500, 96), act(500, 64), out) >= 500 * 64 * 2          # the decoded input at least
    assert size(mat(500, 96, dtype=_abi.ISO_F32), act(500, 64), out) >= 500 * (64 + 3 * 96) * 2
    assert size(mat(1, 96), act(1, 64), out) < 4096                       # few tokens need none
    assert size(mat(500, 96), act(501, 64), out) == _abi.ISO_ERR_SHAPE
    assert size(mat(500, 95), act(500, 64), out) == _abi.ISO_ERR_SHAPE
    assert size(mat(500, 96), act(500, 32), out) == _abi.ISO_ERR_SHAPE
    assert L.iso_act_wgrad_workspace_size(mat(500, 96), act(500, 64), out, None) == _abi.ISO_ERR_ARG
    assert run(mat(500, 96), act(500, 64), out, acc=2) == _abi.ISO_ERR_ARG
    assert run(mat(500, 96), act(500, 64), out, ws=None) == _abi.ISO_ERR_WORKSPACE
    assert run(mat(500, 96), act(500, 64), out, ws=ctypes.c_void_p(0x40000010)) == _abi.ISO_ERR_WORKSPACE
    need = size(mat(500, 96), act(500, 64), out)
    assert run(mat(500, 96), act(500, 64), out, n=need - 1) == _abi.ISO_ERR_WORKSPACE
    assert run(mat(500, 96), act(500, 64), mat(96, 64, ptr=A)) == _abi.ISO_ERR_ARG          # over dY
    assert run(mat(500, 96), act(500, 64), mat(96, 64, ptr=2 * A)) == _abi.ISO_ERR_ARG      # over the codes
    assert run(mat(500, 96), act(500, 64), mat(96, 64, ptr=3 * A)) == _abi.ISO_ERR_ARG      # over the exponents
    assert run(mat(500, 96), act(500, 64), mat(96, 64, ptr=6 * A, dtype=5)) == _abi.ISO_ERR_DTYPE


def test_embedding_refusals():
    L = _abi.lib()
    nb = ctypes.c_size_t()
    ids = ctypes.c_void_p(7 * A)

    def embed(table, out, ids=ids, i64=1, n=8, scale=1.0):
        return L.iso_embed(table, ids, i64, n, -1, scale, out, None, None)

    def grad(dy, g, ids=ids, i64=1, scale=1.0, acc=0, ws=WS, n=BIG):
        return L.iso_embed_grad(dy, ids, i64, -1, scale, g, acc, ws, n, None, None)
    t, o = mat(50, 64), mat(8, 64, ptr=6 * A)
    assert embed(t, mat(9, 64, ptr=6 * A)) == _abi.ISO_ERR_SHAPE
    assert embed(t, mat(8, 63, ptr=6 * A)) == _abi.ISO_ERR_SHAPE
    assert embed(t, o, scale=float("inf")) == _abi.ISO_ERR_ARG
    assert embed(t, o, i64=2) == _abi.ISO_ERR_ARG
    assert embed(t, o, ids=None) == _abi.ISO_ERR_ARG
    assert embed(t, o, ids=ctypes.c_void_p(7 * A + 4)) == _abi.ISO_ERR_ALIGN
    assert embed(t, mat(8, 64, ptr=A + 128)) == _abi.ISO_ERR_ARG
    assert embed(t, mat(8, 64, ptr=7 * A)) == _abi.ISO_ERR_ARG                # over the ids
    assert embed(t, mat(0, 64, ptr=None), ids=None, n=0) == _abi.ISO_OK
    dy, g = mat(8, 64), mat(50, 64, ptr=6 * A, dtype=_abi.ISO_F32)
    assert grad(dy, mat(50, 63, ptr=6 * A)) == _abi.ISO_ERR_SHAPE
    assert grad(dy, g, scale=float("nan")) == _abi.ISO_ERR_ARG
    assert grad(dy, g, acc=-1) == _abi.ISO_ERR_ARG
    assert grad(dy, g, ws=None) == _abi.ISO_ERR_WORKSPACE
    assert grad(dy, g, n=16) == _abi.ISO_ERR_WORKSPACE
    assert grad(dy, mat(50, 64, ptr=A)) == _abi.ISO_ERR_ARG
    assert grad(dy, mat(50, 64, ptr=7 * A - 64)) == _abi.ISO_ERR_ARG
    assert L.iso_embed_grad_workspace_size(-1, 64, nb) == _abi.ISO_ERR_SHAPE
    assert L.iso_embed_grad_workspace_size(1 << 31, 64, nb) == _abi.ISO_ERR_UNSUPPORTED
    assert L.iso_embed_grad_workspace_size(5000, 64, nb) == _abi.ISO_OK and nb.value >= 2 * 8 * 5000


def test_python_checks_without_a_gpu():
    with pytest.raises(ValueError, match="CUDA"):
        iso.act_pack(torch.zeros(4, 64, dtype=torch.bfloat16))
    with pytest.raises(TypeError, match="bfloat16 or float32"):
        iso.act_pack(torch.zeros(4, 64, dtype=torch.float16))
    with pytest.raises(ValueError, match="2-D"):
        iso.act_pack(torch.zeros(4, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="CUDA"):
        iso.ActPack(torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4, 8, dtype=torch.uint8), 64)
    with pytest.raises(TypeError):
        iso.ActPack(torch.zeros(4, 64), torch.zeros(4, 8, dtype=torch.uint8), 64)
    with pytest.raises(TypeError, match="int32 or int64"):
        iso.train._ids(torch.zeros(4))
