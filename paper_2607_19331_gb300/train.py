"""PyTorch-facing binding of the training-step operators (include/iso.h):
8-bit activation checkpoints, the weight and SwiGLU gradients taken from them,
and the token embedding with its gradient.

Argument marshalling only, as in ``api``; every step of the computation runs in
libiso_gb300.so.  Matrices are 2-D CUDA tensors (tokens in rows), bfloat16 or
float32, with unit stride along a row and any row stride.  Work is enqueued on
``stream`` (default: the current stream), where tensors that a call allocates
belong too; nothing waits for the device.
"""
from __future__ import annotations

import ctypes
import math
from dataclasses import dataclass
from typing import Optional, Tuple

import torch

from . import _abi
from ._abi import IsoAct, IsoMat, check, lib
from .api import Workspace

GROUP = _abi.ISO_ACT_GROUP
_CODES = {torch.bfloat16: _abi.ISO_BF16, torch.float32: _abi.ISO_F32}


def _mat(t: torch.Tensor, name: str) -> IsoMat:
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D tensor")
    if t.dtype not in _CODES:
        raise TypeError(f"{name} must be bfloat16 or float32, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    rows, cols = t.shape
    ld, unit = t.stride()
    if cols > 1 and unit != 1:
        raise ValueError(f"{name} must have unit stride along its rows")
    if rows <= 1 or cols == 0:
        ld = max(ld, cols)
    if ld < cols:
        raise ValueError(f"{name} has overlapping rows")
    return IsoMat(t.data_ptr(), rows, cols, ld, _CODES[t.dtype], 0)


def _same_device(first: torch.Tensor, *rest: Optional[torch.Tensor]) -> torch.device:
    dev = first.device
    for t in rest:
        if t is not None and t.device != dev:
            raise ValueError(f"tensors on different devices: {dev} and {t.device}")
    return dev


class _On:
    """The stream of a call.  Given explicitly, tensors are allocated on it
    while the call runs, so that their memory is not reused before its work."""

    def __init__(self, dev: torch.device, stream):
        if torch.cuda.current_device() != dev.index:
            raise ValueError(f"tensors are on {dev}, the current device is cuda:{torch.cuda.current_device()}")
        self.ctx = None
        if stream is not None:
            self.ctx = torch.cuda.stream(stream)
        else:
            stream = torch.cuda.current_stream(dev)
        self.ptr = stream.cuda_stream

    def __enter__(self):
        if self.ctx is not None:
            self.ctx.__enter__()
        return self.ptr

    def __exit__(self, *exc):
        if self.ctx is not None:
            self.ctx.__exit__(*exc)
        return False


_workspaces = {}


def _workspace(ws: Optional[Workspace], dev: torch.device, stream_ptr: int) -> Workspace:
    """The caller's workspace, or a default one of the call's own stream (calls
    on different streams may overlap and must not share scratch)."""
    if ws is not None:
        return ws
    key = (dev.index, stream_ptr)
    got = _workspaces.get(key)
    if got is None:
        got = _workspaces[key] = Workspace(dev)
    return got


def _status(want: bool, dev):
    return torch.zeros(1, dtype=torch.int32, device=dev) if want else None


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


# ---------------------------------------------------------------------------
# checkpoints
# ---------------------------------------------------------------------------
@dataclass
class ActPack:
    """A matrix kept in 8 bits (iso_act): int8 codes and one exponent byte per
    32 channels, 1.03 bytes an entry.  ``dtype`` is the packed matrix's type,
    the default of act_unpack.  ``rows(a, b)`` is the checkpoint of a range of
    rows, sharing storage."""
    codes: torch.Tensor   # int8 [rows, cols rounded up to 32]
    exps: torch.Tensor    # uint8 [rows, groups rounded up to 8]
    cols: int
    dtype: torch.dtype = torch.bfloat16

    @staticmethod
    def empty(rows: int, cols: int, dtype=torch.bfloat16, device="cuda") -> "ActPack":
        groups = -(-cols // GROUP)
        return ActPack(torch.empty(rows, groups * GROUP, dtype=torch.int8, device=device),
                       torch.empty(rows, -(-groups // 8) * 8, dtype=torch.uint8, device=device), cols, dtype)

    @property
    def shape(self) -> Tuple[int, int]:
        return int(self.codes.shape[0]), self.cols

    @property
    def nbytes(self) -> int:
        return self.codes.numel() + self.exps.numel()

    def rows(self, a: int, b: int) -> "ActPack":
        return ActPack(self.codes[a:b], self.exps[a:b], self.cols, self.dtype)

    def abi(self) -> IsoAct:
        c, e = self.codes, self.exps
        if c.dtype != torch.int8 or e.dtype != torch.uint8 or c.dim() != 2 or e.dim() != 2:
            raise TypeError("a checkpoint holds 2-D int8 codes and uint8 exponents")
        if not c.is_cuda or e.device != c.device:
            raise ValueError("a checkpoint's codes and exponents must be on one CUDA device")
        groups = -(-self.cols // GROUP)
        if c.shape[0] != e.shape[0] or c.shape[1] < groups * GROUP or e.shape[1] < -(-groups // 8) * 8:
            raise ValueError("a checkpoint's codes and exponents do not fit its shape")
        if self.cols and (c.stride(1) != 1 or e.stride(1) != 1):
            raise ValueError("a checkpoint's codes and exponents must have unit stride along their rows")
        one = c.shape[0] <= 1
        return IsoAct(c.data_ptr(), e.data_ptr(), c.shape[0], self.cols, c.shape[1] if one else c.stride(0),
                      e.shape[1] if one else e.stride(0))


def act_pack(x: torch.Tensor, out: Optional[ActPack] = None, stream=None) -> ActPack:
    """The 8-bit checkpoint of x (iso_act_pack)."""
    dx = _mat(x, "x")
    with _On(x.device, stream) as s:
        if out is None:
            out = ActPack.empty(dx.rows, dx.cols, x.dtype, x.device)
        _same_device(x, out.codes)
        check(lib().iso_act_pack(dx, out.abi(), s), "iso_act_pack")
    return out


def act_unpack(pack: ActPack, dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
               stream=None) -> torch.Tensor:
    """The values a checkpoint stands for (iso_act_unpack), exact in either type."""
    dp = pack.abi()
    with _On(pack.codes.device, stream) as s:
        if out is None:
            out = torch.empty(pack.shape, dtype=dtype or pack.dtype, device=pack.codes.device)
        elif dtype is not None and out.dtype != dtype:
            raise TypeError(f"out is {out.dtype}, dtype asks for {dtype}")
        _same_device(pack.codes, out)
        check(lib().iso_act_unpack(dp, _mat(out, "out"), s), "iso_act_unpack")
    return out


def act_wgrad_workspace_size(dy: torch.Tensor, pack: ActPack, out: torch.Tensor) -> int:
    nb = ctypes.c_size_t(0)
    check(lib().iso_act_wgrad_workspace_size(_mat(dy, "dy"), pack.abi(), _mat(out, "out"), nb),
          "iso_act_wgrad_workspace_size")
    return int(nb.value)


def act_wgrad(dy: torch.Tensor, pack: ActPack, out: Optional[torch.Tensor] = None, dtype=torch.float32,
              accumulate=False, workspace: Optional[Workspace] = None, status=False, stream=None):
    """The weight gradient dy^T x_hat of y = x W^T from x's checkpoint
    (iso_act_wgrad), out_features x in_features, as opt_step takes it; added to
    ``out`` with accumulate.  Returns out (and the device status with
    status=True)."""
    if accumulate and out is None:
        raise ValueError("accumulate needs an out to add to")
    dd, dp = _mat(dy, "dy"), pack.abi()
    dev = _same_device(dy, pack.codes, out)
    with _On(dev, stream) as s:
        if out is None:
            out = torch.empty(dd.cols, dp.cols, dtype=dtype, device=dev)
        do = _mat(out, "out")
        nb = ctypes.c_size_t(0)
        check(lib().iso_act_wgrad_workspace_size(dd, dp, do, nb), "iso_act_wgrad")
        wptr, wlen = _workspace(workspace, dev, s).get(nb.value)
        st = _status(status, dev)
        check(lib().iso_act_wgrad(dd, dp, do, int(bool(accumulate)), wptr, wlen, _ptr(st), s), "iso_act_wgrad")
    return (out, st) if status else out


# ---------------------------------------------------------------------------
# SwiGLU
# ---------------------------------------------------------------------------
def swiglu_pack(gate: torch.Tensor, up: torch.Tensor, out: Optional[torch.Tensor] = None,
                packs: Optional[Tuple[ActPack, ActPack]] = None, stream=None):
    """(h, gate_pack, up_pack): h = silu(gate) up and the checkpoints of both
    inputs in one pass (iso_swiglu_pack).  gate and up may be the halves of
    one buffer."""
    dg, du = _mat(gate, "gate"), _mat(up, "up")
    dev = _same_device(gate, up, out)
    with _On(dev, stream) as s:
        if out is None:
            out = torch.empty(gate.shape, dtype=gate.dtype, device=dev)
        if packs is None:
            packs = (ActPack.empty(dg.rows, dg.cols, gate.dtype, dev), ActPack.empty(du.rows, du.cols, up.dtype, dev))
        _same_device(gate, packs[0].codes, packs[1].codes)
        check(lib().iso_swiglu_pack(dg, du, _mat(out, "out"), packs[0].abi(), packs[1].abi(), s), "iso_swiglu_pack")
    return out, packs[0], packs[1]


def swiglu_grad(dh: torch.Tensor, gate_pack: ActPack, up_pack: ActPack, out=None, need_h=True, stream=None):
    """(d_gate, d_up, h) from the gradient of h and the checkpoints of its
    inputs (iso_swiglu_grad); h is None without need_h.  ``out`` gives the
    tensors to write, d_gate and d_up possibly the halves of one buffer."""
    dd, pg, pu = _mat(dh, "dh"), gate_pack.abi(), up_pack.abi()
    dev = _same_device(dh, gate_pack.codes, up_pack.codes)
    with _On(dev, stream) as s:
        if out is None:
            out = [torch.empty(dh.shape, dtype=dh.dtype, device=dev) for _ in range(3 if need_h else 2)]
        d_gate, d_up = out[0], out[1]
        h = out[2] if need_h else None
        _same_device(dh, d_gate, d_up, h)
        check(lib().iso_swiglu_grad(dd, pg, pu, _mat(d_gate, "d_gate"), _mat(d_up, "d_up"),
                                    _mat(h, "h") if need_h else None, s), "iso_swiglu_grad")
    return d_gate, d_up, h


# ---------------------------------------------------------------------------
# token embedding
# ---------------------------------------------------------------------------
def _ids(ids: torch.Tensor):
    if not isinstance(ids, torch.Tensor) or ids.dtype not in (torch.int32, torch.int64):
        raise TypeError("ids must be an int32 or int64 tensor")
    if not ids.is_cuda or not ids.is_contiguous():
        raise ValueError("ids must be a contiguous CUDA tensor")
    return ids.data_ptr(), int(ids.dtype == torch.int64), ids.numel()


def _scale(scale) -> float:
    scale = float(scale)
    if not math.isfinite(scale):
        raise ValueError("scale must be finite")
    return scale


def embed(table: torch.Tensor, ids: torch.Tensor, scale=1.0, pad_id: Optional[int] = None,
          out: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None, status=False, stream=None):
    """scale * table[ids] (iso_embed), one row per id in ids' flat order; zero
    rows where the id is pad_id.  Other ids outside the table give zero rows
    and ISO_ERR_INDEX in the device status (returned with status=True)."""
    dt = _mat(table, "table")
    ptr, i64, n = _ids(ids)
    dev = _same_device(table, ids, out)
    with _On(dev, stream) as s:
        if out is None:
            out = torch.empty(n, dt.cols, dtype=dtype or table.dtype, device=dev)
        elif dtype is not None and out.dtype != dtype:
            raise TypeError(f"out is {out.dtype}, dtype asks for {dtype}")
        st = _status(status, dev)
        check(lib().iso_embed(dt, ptr, i64, n, -1 if pad_id is None else int(pad_id), _scale(scale),
                              _mat(out, "out"), _ptr(st), s), "iso_embed")
    return (out, st) if status else out


def embed_grad_workspace_size(n: int, cols: int) -> int:
    nb = ctypes.c_size_t(0)
    check(lib().iso_embed_grad_workspace_size(int(n), int(cols), nb), "iso_embed_grad_workspace_size")
    return int(nb.value)


def embed_grad(dy: torch.Tensor, ids: torch.Tensor, rows: Optional[int] = None, scale=1.0,
               pad_id: Optional[int] = None, out: Optional[torch.Tensor] = None, dtype=torch.float32,
               accumulate=False, workspace: Optional[Workspace] = None, status=False, stream=None):
    """The gradient of embed's table (iso_embed_grad): rows x cols, zero where
    no token has the row's id; added to ``out`` with accumulate.  The same
    inputs give the same bits.  Returns out (and the device status with
    status=True)."""
    if accumulate and out is None:
        raise ValueError("accumulate needs an out to add to")
    if out is None and rows is None:
        raise ValueError("embed_grad needs rows (the table's) or out")
    dd = _mat(dy, "dy")
    ptr, i64, n = _ids(ids)
    if n != dd.rows:
        raise ValueError(f"{n} ids for {dd.rows} rows of dy")
    if out is not None and rows is not None and out.shape[0] != rows:
        raise ValueError(f"out has {out.shape[0]} rows, rows is {rows}")
    dev = _same_device(dy, ids, out)
    with _On(dev, stream) as s:
        if out is None:
            out = torch.empty(rows, dd.cols, dtype=dtype, device=dev)
        wptr, wlen = _workspace(workspace, dev, s).get(embed_grad_workspace_size(n, dd.cols))
        st = _status(status, dev)
        check(lib().iso_embed_grad(dd, ptr, i64, -1 if pad_id is None else int(pad_id), _scale(scale),
                                   _mat(out, "out"), int(bool(accumulate)), wptr, wlen, _ptr(st), s),
              "iso_embed_grad")
    return (out, st) if status else out
