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
import functools
import math
from typing import Optional, Tuple

import torch

from . import _abi
from ._abi import IsoAct, IsoMat, check, lib
from .api import Workspace

GROUP = _abi.ISO_ACT_GROUP
_CODES = {torch.bfloat16: _abi.ISO_BF16, torch.float32: _abi.ISO_F32}
_byref = ctypes.byref
# the current stream's handle without a Stream object, where this torch has it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _mat(t: torch.Tensor, name: str) -> IsoMat:
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D tensor")
    code = _CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be bfloat16 or float32, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    rows, cols = t.shape
    ld, unit = t.stride()
    if unit != 1 and cols > 1:
        raise ValueError(f"{name} must have unit stride along its rows")
    if ld < cols:
        if rows > 1 and cols:
            raise ValueError(f"{name} has overlapping rows")
        ld = cols
    return IsoMat(t.data_ptr(), rows, cols, ld, code, 0)


def _new(rows: int, cols: int, dtype, device):
    """A new contiguous matrix and its descriptor."""
    code = _CODES.get(dtype)
    if code is None:
        raise TypeError(f"tensors must be bfloat16 or float32, got {dtype}")
    t = torch.empty((rows, cols), dtype=dtype, device=device)
    return t, IsoMat(t.data_ptr(), rows, cols, cols, code, 0)


class _On:
    """The stream and device of a call, from its first tensor: ``s`` is the raw
    stream.  Entered, an explicit stream is the current one, so that tensors
    allocated meanwhile belong to it and their memory is not reused before its
    work.  The tensors' device must be the current one."""

    __slots__ = ("s", "index", "device", "ctx")

    def __init__(self, first: torch.Tensor, stream):
        self.device = first.device
        self.index = first.get_device()
        if torch.cuda.current_device() != self.index:
            raise ValueError(f"tensors are on {self.device}, the current device is cuda:{torch.cuda.current_device()}")
        if stream is None:
            self.ctx = None
            self.s = _raw_stream(self.index)
        else:
            self.ctx = torch.cuda.stream(stream)
            self.s = stream.cuda_stream

    def __enter__(self):
        if self.ctx is not None:
            self.ctx.__enter__()
        return self

    def __exit__(self, *exc):
        if self.ctx is not None:
            self.ctx.__exit__(*exc)
        return False

    def has(self, *tensors: Optional[torch.Tensor]):
        for t in tensors:
            if t is not None and t.get_device() != self.index:
                raise ValueError(f"tensors on different devices: {self.device} and {t.device}")


_workspaces = {}


def _scratch(ws: Optional[Workspace], on: _On, nbytes: int):
    """The caller's workspace, or a default one of the call's own stream (calls
    on different streams may overlap and must not share scratch)."""
    if ws is None:
        key = (on.index, on.s)
        ws = _workspaces.get(key)
        if ws is None:
            ws = _workspaces[key] = Workspace(on.device)
    return ws.get(nbytes)


def _status(want: bool, device):
    return torch.zeros(1, dtype=torch.int32, device=device) if want else None


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


# ---------------------------------------------------------------------------
# checkpoints
# ---------------------------------------------------------------------------
class ActPack:
    """A matrix kept in 8 bits (iso_act): int8 codes [rows, cols rounded up to
    32] and one exponent byte per 32 channels (uint8 [rows, groups rounded up
    to 8]), 1.03 bytes an entry.  ``dtype`` is the packed matrix's type, the
    default of act_unpack.  ``rows(a, b)`` is the checkpoint of a range of
    rows, sharing storage."""

    __slots__ = ("cols", "dtype", "_abi", "_parts", "_buf")

    def __init__(self, codes: torch.Tensor, exps: torch.Tensor, cols: int, dtype=torch.bfloat16):
        if codes.dtype != torch.int8 or exps.dtype != torch.uint8 or codes.dim() != 2 or exps.dim() != 2:
            raise TypeError("a checkpoint holds 2-D int8 codes and uint8 exponents")
        if not codes.is_cuda or exps.device != codes.device:
            raise ValueError("a checkpoint's codes and exponents must be on one CUDA device")
        if dtype not in _CODES:
            raise TypeError(f"a checkpoint's dtype must be bfloat16 or float32, got {dtype}")
        groups = -(-cols // GROUP)
        if codes.shape[0] != exps.shape[0] or codes.shape[1] < groups * GROUP or exps.shape[1] < -(-groups // 8) * 8:
            raise ValueError("a checkpoint's codes and exponents do not fit its shape")
        if cols and (codes.stride(1) != 1 or exps.stride(1) != 1):
            raise ValueError("a checkpoint's codes and exponents must have unit stride along their rows")
        rows, one = codes.shape[0], codes.shape[0] <= 1
        self.cols, self.dtype, self._buf, self._parts = cols, dtype, codes, (codes, exps)
        self._abi = IsoAct(codes.data_ptr(), exps.data_ptr(), rows, cols, codes.shape[1] if one else codes.stride(0),
                           exps.shape[1] if one else exps.stride(0))

    @staticmethod
    def empty(rows: int, cols: int, dtype=torch.bfloat16, device="cuda") -> "ActPack":
        """Uninitialised storage (one buffer, the codes first) for act_pack's
        and swiglu_pack's outputs."""
        if dtype not in _CODES:
            raise TypeError(f"a checkpoint's dtype must be bfloat16 or float32, got {dtype}")
        groups = -(-cols // GROUP)
        ldc, lde = groups * GROUP, -(-groups // 8) * 8
        self = object.__new__(ActPack)
        self.cols, self.dtype, self._parts = cols, dtype, None
        self._buf = buf = torch.empty(rows * (ldc + lde), dtype=torch.uint8, device=device)
        at = buf.data_ptr()
        self._abi = IsoAct(at, at + rows * ldc, rows, cols, ldc, lde)
        return self

    def _views(self):
        if self._parts is None:
            a = self._abi
            n = a.rows * a.ld_codes
            self._parts = (self._buf[:n].view(torch.int8).view(a.rows, a.ld_codes),
                           self._buf[n:].view(a.rows, a.ld_exps))
        return self._parts

    @property
    def codes(self) -> torch.Tensor:
        return self._views()[0]

    @property
    def exps(self) -> torch.Tensor:
        return self._views()[1]

    @property
    def shape(self) -> Tuple[int, int]:
        return self._abi.rows, self.cols

    @property
    def nbytes(self) -> int:
        return self.codes.numel() + self.exps.numel()

    def rows(self, a: int, b: int) -> "ActPack":
        return ActPack(self.codes[a:b], self.exps[a:b], self.cols, self.dtype)

    def __repr__(self):
        return f"ActPack(shape={self.shape}, dtype={self.dtype}, device={self._buf.device})"


def act_pack(x: torch.Tensor, out: Optional[ActPack] = None, stream=None) -> ActPack:
    """The 8-bit checkpoint of x (iso_act_pack)."""
    dx = _mat(x, "x")
    with _On(x, stream) as on:
        if out is None:
            out = ActPack.empty(dx.rows, dx.cols, x.dtype, on.device)
        else:
            on.has(out._buf)
        check(lib().iso_act_pack(_byref(dx), _byref(out._abi), on.s), "iso_act_pack")
    return out


def act_unpack(pack: ActPack, dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
               stream=None) -> torch.Tensor:
    """The values a checkpoint stands for (iso_act_unpack), exact in either type."""
    with _On(pack._buf, stream) as on:
        if out is None:
            out, do = _new(pack._abi.rows, pack.cols, dtype or pack.dtype, on.device)
        else:
            if dtype is not None and out.dtype != dtype:
                raise TypeError(f"out is {out.dtype}, dtype asks for {dtype}")
            do = _mat(out, "out")
            on.has(out)
        check(lib().iso_act_unpack(_byref(pack._abi), _byref(do), on.s), "iso_act_unpack")
    return out


def act_wgrad_workspace_size(dy: torch.Tensor, pack: ActPack, out: torch.Tensor) -> int:
    nb = ctypes.c_size_t(0)
    check(lib().iso_act_wgrad_workspace_size(_byref(_mat(dy, "dy")), _byref(pack._abi), _byref(_mat(out, "out")),
                                             _byref(nb)), "iso_act_wgrad_workspace_size")
    return int(nb.value)


def act_wgrad(dy: torch.Tensor, pack: ActPack, out: Optional[torch.Tensor] = None, dtype=None, accumulate=False,
              workspace: Optional[Workspace] = None, status=False, stream=None):
    """The weight gradient dy^T x_hat of y = x W^T from x's checkpoint
    (iso_act_wgrad), out_features x in_features, as opt_step takes it, in
    ``dtype`` (float32) or into ``out``; added to ``out`` with accumulate.
    Returns it (and the device status with status=True)."""
    dd = _mat(dy, "dy")
    with _On(dy, stream) as on:
        on.has(pack._buf)
        if out is None:
            if accumulate:
                raise ValueError("accumulate needs an out to add to")
            out, do = _new(dd.cols, pack.cols, dtype or torch.float32, on.device)
        else:
            if dtype is not None and out.dtype != dtype:
                raise TypeError(f"out is {out.dtype}, dtype asks for {dtype}")
            do = _mat(out, "out")
            on.has(out)
        nb = ctypes.c_size_t(0)
        check(lib().iso_act_wgrad_workspace_size(_byref(dd), _byref(pack._abi), _byref(do), _byref(nb)), "iso_act_wgrad")
        wptr, wlen = _scratch(workspace, on, nb.value)
        st = _status(status, on.device)
        check(lib().iso_act_wgrad(_byref(dd), _byref(pack._abi), _byref(do), int(bool(accumulate)), wptr, wlen,
                                  _ptr(st), on.s), "iso_act_wgrad")
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
    with _On(gate, stream) as on:
        on.has(up)
        if out is None:
            out, do = _new(dg.rows, dg.cols, gate.dtype, on.device)
        else:
            do = _mat(out, "out")
            on.has(out)
        if packs is None:
            packs = (ActPack.empty(dg.rows, dg.cols, gate.dtype, on.device),
                     ActPack.empty(dg.rows, dg.cols, gate.dtype, on.device))
        else:
            on.has(packs[0]._buf, packs[1]._buf)
        check(lib().iso_swiglu_pack(_byref(dg), _byref(du), _byref(do), _byref(packs[0]._abi), _byref(packs[1]._abi),
                                    on.s), "iso_swiglu_pack")
    return out, packs[0], packs[1]


def swiglu_grad(dh: torch.Tensor, gate_pack: ActPack, up_pack: ActPack, out=None, need_h=True, stream=None):
    """(d_gate, d_up, h) from the gradient of h and the checkpoints of its
    inputs (iso_swiglu_grad); h is None without need_h.  ``out`` gives the
    tensors to write, d_gate and d_up possibly the halves of one buffer."""
    dd = _mat(dh, "dh")
    n = 3 if need_h else 2
    with _On(dh, stream) as on:
        on.has(gate_pack._buf, up_pack._buf)
        if out is None:
            got = [_new(dd.rows, dd.cols, dh.dtype, on.device) for _ in range(n)]
            out, descs = [g[0] for g in got], [g[1] for g in got]
        else:
            if len(out) < n:
                raise ValueError(f"out needs {n} tensors")
            descs = [_mat(t, w) for t, w in zip(out[:n], ("d_gate", "d_up", "h"))]
            on.has(*out[:n])
        check(lib().iso_swiglu_grad(_byref(dd), _byref(gate_pack._abi), _byref(up_pack._abi), _byref(descs[0]),
                                    _byref(descs[1]), _byref(descs[2]) if need_h else None, on.s), "iso_swiglu_grad")
    return out[0], out[1], out[2] if need_h else None


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
    """scale * table[ids] (iso_embed), one row per id in ids' flat order, in the
    table's type unless ``dtype`` or ``out`` says otherwise; zero rows where
    the id is pad_id.  Other ids outside the table give zero rows and
    ISO_ERR_INDEX in the device status (returned with status=True)."""
    dt = _mat(table, "table")
    ptr, i64, n = _ids(ids)
    with _On(table, stream) as on:
        on.has(ids)
        if out is None:
            out, do = _new(n, dt.cols, dtype or table.dtype, on.device)
        else:
            if dtype is not None and out.dtype != dtype:
                raise TypeError(f"out is {out.dtype}, dtype asks for {dtype}")
            do = _mat(out, "out")
            on.has(out)
        st = _status(status, on.device)
        check(lib().iso_embed(_byref(dt), ptr, i64, n, -1 if pad_id is None else int(pad_id), _scale(scale),
                              _byref(do), _ptr(st), on.s), "iso_embed")
    return (out, st) if status else out


@functools.lru_cache(maxsize=64)
def embed_grad_workspace_size(n: int, cols: int) -> int:
    nb = ctypes.c_size_t(0)
    check(lib().iso_embed_grad_workspace_size(int(n), int(cols), _byref(nb)), "iso_embed_grad_workspace_size")
    return int(nb.value)


def embed_grad(dy: torch.Tensor, ids: torch.Tensor, rows: Optional[int] = None, scale=1.0,
               pad_id: Optional[int] = None, out: Optional[torch.Tensor] = None, dtype=None, accumulate=False,
               workspace: Optional[Workspace] = None, status=False, stream=None):
    """The gradient of embed's table (iso_embed_grad), rows x cols in ``dtype``
    (float32) or into ``out``, zero where no token has the row's id; added to
    ``out`` with accumulate.  The same inputs give the same bits.  Returns it
    (and the device status with status=True)."""
    dd = _mat(dy, "dy")
    ptr, i64, n = _ids(ids)
    if n != dd.rows:
        raise ValueError(f"{n} ids for {dd.rows} rows of dy")
    with _On(dy, stream) as on:
        on.has(ids)
        if out is None:
            if accumulate:
                raise ValueError("accumulate needs an out to add to")
            if rows is None:
                raise ValueError("embed_grad needs rows (the table's) or out")
            out, do = _new(int(rows), dd.cols, dtype or torch.float32, on.device)
        else:
            if rows is not None and out.shape[0] != rows:
                raise ValueError(f"out has {out.shape[0]} rows, rows is {rows}")
            if dtype is not None and out.dtype != dtype:
                raise TypeError(f"out is {out.dtype}, dtype asks for {dtype}")
            do = _mat(out, "out")
            on.has(out)
        wptr, wlen = _scratch(workspace, on, embed_grad_workspace_size(n, dd.cols))
        st = _status(status, on.device)
        check(lib().iso_embed_grad(_byref(dd), ptr, i64, -1 if pad_id is None else int(pad_id), _scale(scale),
                                   _byref(do), int(bool(accumulate)), wptr, wlen, _ptr(st), on.s), "iso_embed_grad")
    return (out, st) if status else out
