"""PyTorch-facing binding of the training-step operators (include/iso.h):
8-bit activation checkpoints, the weight and SwiGLU gradients taken from them,
and the token embedding with its gradient.

Argument marshalling only, as in ``api``; every step of the computation runs in
libiso_gb300.so.  The common form of a call (outputs allocated by it, on the
current stream) is marshalled by the host module ``_iso_train``
(csrc/train_binding.cpp), any other form here.  Matrices are 2-D CUDA tensors
(tokens in rows), bfloat16 or float32, with unit stride along a row and any row
stride.  Work is enqueued on ``stream`` (default: the current stream), where
tensors that a call allocates belong too; nothing waits for the device.  The
calls stand outside autograd: inputs that require a gradient are taken as they
are and results carry no graph; gradients come from the calls that name them.
"""
from __future__ import annotations

import ctypes
import functools
import importlib.util
import math
from typing import Optional, Tuple

import torch

from . import _abi, build
from ._abi import IsoAct, IsoMat, check, lib
from .api import Workspace

GROUP = _abi.ISO_ACT_GROUP
_CODES = {torch.bfloat16: _abi.ISO_BF16, torch.float32: _abi.ISO_F32}
_byref = ctypes.byref
_native = None


def _load_native():
    """The host module beside the loaded library; raises if it has not been built,
    or was built for another torch."""
    global _native
    if _native is None:
        lib()
        path, made_for = build.BINDING, build.stamped_torch()
        if made_for != torch.__version__:
            raise RuntimeError((f"_iso_train not found at {path}" if made_for is None else
                                f"{path} was built for torch {made_for}, this is torch {torch.__version__}") +
                               ": build it first (python -c 'import __graft_entry__ as g; g.build()')")
        spec = importlib.util.spec_from_file_location("_iso_train", path)
        mod = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(mod)
        _native = mod
    return _native
# the current stream's handle without a Stream object, where this torch has it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _mat(t: torch.Tensor, name: str) -> IsoMat:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor")
    if t.dim() != 2:
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


def _here(first: torch.Tensor, *rest: Optional[torch.Tensor]) -> int:
    """The current stream's handle; the tensors must be on the current device."""
    index = first.get_device()
    if torch.cuda.current_device() != index:
        raise ValueError(f"tensors are on {first.device}, the current device is cuda:{torch.cuda.current_device()}")
    for t in rest:
        if t is not None and t.get_device() != index:
            raise ValueError(f"tensors on different devices: {first.device} and {t.device}")
    return _raw_stream(index)


def _scratch(ws: Optional[Workspace], device: torch.device) -> Workspace:
    """The caller's workspace, or one for this call alone, from torch's allocator
    on the current stream: calls of several threads on one stream may interleave
    their launches, and a captured call's scratch belongs to its graph.  To be
    held until the call is enqueued."""
    return Workspace(device) if ws is None else ws


def _done(result, where: str):
    """The native call's result, or the error its status code stands for."""
    if type(result) is int:
        check(result, where)
    return result


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

    # _t: storage, addresses of codes and exponents, rows, cols, row strides of both
    __slots__ = ("dtype", "_t", "_parts")

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
        one = codes.shape[0] <= 1
        self.dtype, self._parts = dtype, (codes, exps)
        self._t = (codes, codes.data_ptr(), exps.data_ptr(), int(codes.shape[0]), int(cols),
                   int(codes.shape[1]) if one else codes.stride(0), int(exps.shape[1]) if one else exps.stride(0))

    @staticmethod
    def _of(t: tuple, dtype) -> "ActPack":
        self = object.__new__(ActPack)
        self.dtype, self._t, self._parts = dtype, t, None
        return self

    @staticmethod
    def empty(rows: int, cols: int, dtype=torch.bfloat16, device="cuda") -> "ActPack":
        """Uninitialised storage (one buffer, the codes first) for act_pack's
        and swiglu_pack's outputs."""
        if dtype not in _CODES:
            raise TypeError(f"a checkpoint's dtype must be bfloat16 or float32, got {dtype}")
        groups = -(-cols // GROUP)
        ldc, lde = groups * GROUP, -(-groups // 8) * 8
        buf = torch.empty(rows * (ldc + lde), dtype=torch.uint8, device=device)
        at = buf.data_ptr()
        return ActPack._of((buf, at, at + rows * ldc, rows, cols, ldc, lde), dtype)

    def _views(self):
        if self._parts is None:
            buf, _, _, rows, _, ldc, lde = self._t
            n = rows * ldc
            self._parts = buf[:n].view(torch.int8).view(rows, ldc), buf[n:].view(rows, lde)
        return self._parts

    @property
    def _buf(self) -> torch.Tensor:
        return self._t[0]

    @property
    def _abi(self) -> IsoAct:
        return IsoAct(*self._t[1:])

    @property
    def cols(self) -> int:
        return self._t[4]

    @property
    def codes(self) -> torch.Tensor:
        return self._views()[0]

    @property
    def exps(self) -> torch.Tensor:
        return self._views()[1]

    @property
    def shape(self) -> Tuple[int, int]:
        return self._t[3], self._t[4]

    @property
    def nbytes(self) -> int:
        return self.codes.numel() + self.exps.numel()

    def rows(self, a: int, b: int) -> "ActPack":
        return ActPack(self.codes[a:b], self.exps[a:b], self.cols, self.dtype)

    def __repr__(self):
        return f"ActPack(shape={self.shape}, dtype={self.dtype}, device={self._buf.device})"


# Every entry point, given a stream, runs with it as the current one: tensors
# that the call allocates then belong to it, and their memory is not reused
# before its work.
def act_pack(x: torch.Tensor, out: Optional[ActPack] = None, stream=None) -> ActPack:
    """The 8-bit checkpoint of x (iso_act_pack)."""
    if out is None and stream is None:
        return ActPack._of(_done((_native or _load_native()).act_pack(x), "iso_act_pack"), x.dtype)
    if stream is not None:
        with torch.cuda.stream(stream):
            return act_pack(x, out)
    dx = _mat(x, "x")
    if out is None:
        s = _here(x)
        out = ActPack.empty(dx.rows, dx.cols, x.dtype, x.device)
    else:
        s = _here(x, out._buf)
    check(lib().iso_act_pack(_byref(dx), _byref(out._abi), s), "iso_act_pack")
    return out


def act_unpack(pack: ActPack, dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
               stream=None) -> torch.Tensor:
    """The values a checkpoint stands for (iso_act_unpack), exact in either type."""
    if out is None and stream is None:
        return _done((_native or _load_native()).act_unpack(pack._t, dtype or pack.dtype), "iso_act_unpack")
    if stream is not None:
        with torch.cuda.stream(stream):
            return act_unpack(pack, dtype, out)
    buf = pack._buf
    if out is None:
        s = _here(buf)
        out, do = _new(pack.shape[0], pack.cols, dtype or pack.dtype, buf.device)
    else:
        if dtype is not None and out.dtype != dtype:
            raise TypeError(f"out is {out.dtype}, dtype asks for {dtype}")
        do = _mat(out, "out")
        s = _here(buf, out)
    check(lib().iso_act_unpack(_byref(pack._abi), _byref(do), s), "iso_act_unpack")
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
    if out is None and stream is None and workspace is None and not status and not accumulate:
        return _done((_native or _load_native()).act_wgrad(dy, pack._t, dtype), "iso_act_wgrad")
    if stream is not None:
        with torch.cuda.stream(stream):
            return act_wgrad(dy, pack, out, dtype, accumulate, workspace, status)
    dd = _mat(dy, "dy")
    s = _here(dy, pack._buf, out)
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs an out to add to")
        out, do = _new(dd.cols, pack.cols, dtype or torch.float32, dy.device)
    else:
        if dtype is not None and out.dtype != dtype:
            raise TypeError(f"out is {out.dtype}, dtype asks for {dtype}")
        do = _mat(out, "out")
    ws = _scratch(workspace, dy.device)
    st = _status(status, dy.device)
    L, args, nb = lib(), (_byref(dd), _byref(pack._abi), _byref(do)), ctypes.c_size_t(0)
    check(L.iso_act_wgrad_workspace_size(*args, _byref(nb)), "iso_act_wgrad")
    check(L.iso_act_wgrad(*args, 1 if accumulate else 0, *ws.get(nb.value), _ptr(st), s), "iso_act_wgrad")
    return (out, st) if status else out


# ---------------------------------------------------------------------------
# SwiGLU
# ---------------------------------------------------------------------------
def swiglu_pack(gate: torch.Tensor, up: torch.Tensor, out: Optional[torch.Tensor] = None,
                packs: Optional[Tuple[ActPack, ActPack]] = None, stream=None):
    """(h, gate_pack, up_pack): h = silu(gate) up and the checkpoints of both
    inputs in one pass (iso_swiglu_pack).  gate and up may be the halves of
    one buffer."""
    if out is None and packs is None and stream is None:
        h, a, b = _done((_native or _load_native()).swiglu_pack(gate, up), "iso_swiglu_pack")
        return h, ActPack._of(a, gate.dtype), ActPack._of(b, gate.dtype)
    if stream is not None:
        with torch.cuda.stream(stream):
            return swiglu_pack(gate, up, out, packs)
    dg, du = _mat(gate, "gate"), _mat(up, "up")
    s = _here(gate, up, out)
    if out is None:
        out, do = _new(dg.rows, dg.cols, gate.dtype, gate.device)
    else:
        do = _mat(out, "out")
    if packs is None:
        a = ActPack.empty(dg.rows, dg.cols, gate.dtype, gate.device)
        b = ActPack.empty(dg.rows, dg.cols, gate.dtype, gate.device)
    else:
        a, b = packs
        _here(gate, a._buf, b._buf)
    check(lib().iso_swiglu_pack(_byref(dg), _byref(du), _byref(do), _byref(a._abi), _byref(b._abi), s),
          "iso_swiglu_pack")
    return out, a, b


def swiglu_grad(dh: torch.Tensor, gate_pack: ActPack, up_pack: ActPack, out=None, need_h=True, stream=None):
    """(d_gate, d_up, h) from the gradient of h and the checkpoints of its
    inputs (iso_swiglu_grad); h is None without need_h.  ``out`` gives the
    tensors to write, d_gate and d_up possibly the halves of one buffer."""
    if out is None and stream is None:
        return _done((_native or _load_native()).swiglu_grad(dh, gate_pack._t, up_pack._t, bool(need_h)),
                     "iso_swiglu_grad")
    if stream is not None:
        with torch.cuda.stream(stream):
            return swiglu_grad(dh, gate_pack, up_pack, out, need_h)
    dd = _mat(dh, "dh")
    s = _here(dh, gate_pack._buf, up_pack._buf)
    h = dhh = None
    if out is None:
        rows, cols, dtype, device = dd.rows, dd.cols, dh.dtype, dh.device
        d_gate, dg = _new(rows, cols, dtype, device)
        d_up, du = _new(rows, cols, dtype, device)
        if need_h:
            h, dhh = _new(rows, cols, dtype, device)
    else:
        if len(out) < (3 if need_h else 2):
            raise ValueError("out needs d_gate, d_up and, with need_h, h")
        d_gate, d_up = out[0], out[1]
        dg, du = _mat(d_gate, "d_gate"), _mat(d_up, "d_up")
        if need_h:
            h = out[2]
            dhh = _mat(h, "h")
        _here(dh, d_gate, d_up, h)
    check(lib().iso_swiglu_grad(_byref(dd), _byref(gate_pack._abi), _byref(up_pack._abi), _byref(dg), _byref(du),
                                None if dhh is None else _byref(dhh), s), "iso_swiglu_grad")
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


def _pad(pad_id: Optional[int]) -> int:
    pad_id = -1 if pad_id is None else int(pad_id)
    if not -1 << 63 <= pad_id < 1 << 63:
        raise ValueError("pad_id must fit 64 bits")
    return pad_id


def _rows(rows) -> int:
    if int(rows) < 0:
        raise ValueError("rows must not be negative")
    return int(rows)


def embed(table: torch.Tensor, ids: torch.Tensor, scale=1.0, pad_id: Optional[int] = None,
          out: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None, status=False, stream=None):
    """scale * table[ids] (iso_embed), one row per id in ids' flat order, in the
    table's type unless ``dtype`` or ``out`` says otherwise; zero rows where
    the id is pad_id.  Other ids outside the table give zero rows and
    ISO_ERR_INDEX in the device status (returned with status=True)."""
    if out is None and stream is None and not status:
        return _done((_native or _load_native()).embed(table, ids, _scale(scale), _pad(pad_id),
                                                       dtype), "iso_embed")
    if stream is not None:
        with torch.cuda.stream(stream):
            return embed(table, ids, scale, pad_id, out, dtype, status)
    dt = _mat(table, "table")
    ptr, i64, n = _ids(ids)
    s = _here(table, ids, out)
    if out is None:
        out, do = _new(n, dt.cols, dtype or table.dtype, table.device)
    else:
        if dtype is not None and out.dtype != dtype:
            raise TypeError(f"out is {out.dtype}, dtype asks for {dtype}")
        do = _mat(out, "out")
    st = _status(status, table.device)
    check(lib().iso_embed(_byref(dt), ptr, i64, n, _pad(pad_id), _scale(scale), _byref(do),
                          _ptr(st), s), "iso_embed")
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
    if out is None and rows is not None and stream is None and workspace is None and not status and not accumulate:
        return _done((_native or _load_native()).embed_grad(dy, ids, _rows(rows), _scale(scale),
                                                            _pad(pad_id), dtype),
                     "iso_embed_grad")
    if stream is not None:
        with torch.cuda.stream(stream):
            return embed_grad(dy, ids, rows, scale, pad_id, out, dtype, accumulate, workspace, status)
    dd = _mat(dy, "dy")
    ptr, i64, n = _ids(ids)
    if n != dd.rows:
        raise ValueError(f"{n} ids for {dd.rows} rows of dy")
    s = _here(dy, ids, out)
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs an out to add to")
        if rows is None:
            raise ValueError("embed_grad needs rows (the table's) or out")
        out, do = _new(_rows(rows), dd.cols, dtype or torch.float32, dy.device)
    else:
        if rows is not None and out.shape[0] != rows:
            raise ValueError(f"out has {out.shape[0]} rows, rows is {rows}")
        if dtype is not None and out.dtype != dtype:
            raise TypeError(f"out is {out.dtype}, dtype asks for {dtype}")
        do = _mat(out, "out")
    ws = _scratch(workspace, dy.device)
    wptr, wlen = ws.get(embed_grad_workspace_size(n, dd.cols))
    st = _status(status, dy.device)
    check(lib().iso_embed_grad(_byref(dd), ptr, i64, _pad(pad_id), _scale(scale),
                               _byref(do), 1 if accumulate else 0, wptr, wlen, _ptr(st), s), "iso_embed_grad")
    return (out, st) if status else out
