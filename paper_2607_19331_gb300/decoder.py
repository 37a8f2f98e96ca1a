"""PyTorch-facing binding of the operators between the embedding and the loss of
a training step (include/iso.h): rotary positions, attention over packed
sequences with its gradient, and distillation from a teacher's top logits with
its gradient.

Argument marshalling only, under the rules of ``train``: matrices are 2-D CUDA
tensors with tokens in rows, bfloat16 or float32, with unit stride along a row
and any row stride, so that heads side by side may be column ranges of one
projection's output; work is enqueued on ``stream`` (default: the current
stream), where tensors that a call allocates belong too; nothing waits for the
device, and the calls stand outside autograd.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Sequence, Tuple

import torch

from . import _abi
from ._abi import IsoAttnCfg, IsoMat, IsoRopeCfg, check, lib
from .api import Workspace
from . import train
from .train import _byref, _done, _here, _mat, _new, _ptr, _scratch, _status


def _native():
    return train._native or train._load_native()


def _vector(t: torch.Tensor, name: str, dtype, shape) -> int:
    """The address of a contiguous CUDA tensor of one type and shape."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype:
        raise TypeError(f"{name} must be a {str(dtype).replace('torch.', '')} tensor")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, has {tuple(t.shape)}")
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA tensor")
    return t.data_ptr()


def _integers(t: torch.Tensor, name: str) -> int:
    """1 for an int64 tensor, 0 for an int32 one."""
    if not isinstance(t, torch.Tensor) or t.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"{name} must be an int32 or int64 tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    return int(t.dtype == torch.int64)


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------
class RopePlan:
    """How heads turn by their positions (iso_rope_cfg): per pair of channels an
    angle per position and the axis its position is on.  Made once, by rope_plan."""

    __slots__ = ("head_dim", "rot_dim", "axes", "pairs", "freq", "axis", "_cfg", "_at")

    def __init__(self, head_dim: int, freq: Sequence[float], axis: Sequence[int], axes: int, pairs: str = "halves"):
        if pairs not in ("halves", "neighbours"):
            raise ValueError("pairs must be 'halves' or 'neighbours'")
        if len(freq) != len(axis):
            raise ValueError(f"{len(freq)} angles for {len(axis)} axes")
        n = len(freq)
        if not 1 <= axes <= _abi.ISO_ROPE_MAX_AXES or any(not 0 <= a < axes for a in axis):
            raise ValueError(f"axes must be 1 to {_abi.ISO_ROPE_MAX_AXES}, and every pair's axis one of them")
        if not all(math.isfinite(f) for f in freq):
            raise ValueError("angles must be finite")
        if head_dim < 1 or 2 * n > head_dim or n > _abi.ISO_ROPE_MAX_PAIRS:
            raise ValueError(f"{n} pairs do not fit a head of {head_dim} (or are more than {_abi.ISO_ROPE_MAX_PAIRS})")
        self.head_dim, self.rot_dim, self.axes, self.pairs = int(head_dim), 2 * n, int(axes), pairs
        self.freq, self.axis = (ctypes.c_double * max(n, 1))(*freq), (ctypes.c_int32 * max(n, 1))(*axis)
        # the turn and the turn back, and their addresses
        self._cfg = tuple(IsoRopeCfg(self.head_dim, 2 * n, self.axes, int(pairs == "neighbours"), inverse, 0,
                                     ctypes.addressof(self.freq), ctypes.addressof(self.axis)) for inverse in (0, 1))
        self._at = tuple(ctypes.addressof(c) for c in self._cfg)

    def __repr__(self):
        return f"RopePlan(head_dim={self.head_dim}, rot_dim={self.rot_dim}, axes={self.axes}, pairs={self.pairs!r})"


def rope_plan(head_dim: int, base: float = 10000.0, sections: Optional[Sequence[int]] = None,
              rot_dim: Optional[int] = None, pairs: str = "halves", turns: bool = False,
              per_axis: bool = False) -> RopePlan:
    """The usual plans: pair i of n = rot_dim / 2 (rot_dim: head_dim) turns by
    base^(-i / n) per position.  ``sections`` gives each axis its number of pairs
    (default: one axis), in blocks, or with ``turns`` in turns (axis 0, 1, 2, 0,
    1, 2 ... while an axis has pairs left).  With ``per_axis`` the angles start
    again on each axis: base^(-j / sections[a]) for the j-th pair of axis a."""
    rot_dim = head_dim if rot_dim is None else rot_dim
    if rot_dim < 0 or rot_dim % 2 or rot_dim > head_dim:
        raise ValueError("rot_dim must be even and fit the head")
    if not (base > 0 and math.isfinite(base)):
        raise ValueError("base must be positive and finite")
    n = rot_dim // 2
    sections = (n,) if sections is None else tuple(int(c) for c in sections)
    if not sections or any(c < 0 for c in sections) or sum(sections) != n:
        raise ValueError(f"sections must add up to {n} pairs")
    if turns:
        left, axis = list(sections), []
        while len(axis) < n:
            for a, c in enumerate(left):
                if c:
                    axis.append(a)
                    left[a] -= 1
    else:
        axis = [a for a, c in enumerate(sections) for _ in range(c)]
    seen, freq = [0] * len(sections), []
    for i, a in enumerate(axis):
        freq.append(float(base) ** (-seen[a] / sections[a] if per_axis else -i / n))
        seen[a] += 1
    return RopePlan(head_dim, freq, axis, len(sections), pairs)


def _positions(positions: torch.Tensor, rows: int, axes: int):
    """Address, type, and distance of the axes."""
    i64 = _integers(positions, "positions")
    if tuple(positions.shape) != (axes, rows) and not (axes == 1 and tuple(positions.shape) == (rows,)):
        raise ValueError(f"positions must have shape ({axes}, {rows})" + (f" or ({rows},)" if axes == 1 else "") +
                         f", has {tuple(positions.shape)}")
    if rows > 1 and positions.stride(-1) != 1:
        raise ValueError("positions must be contiguous along an axis")
    ld = positions.stride(0) if positions.dim() == 2 and axes > 1 else rows
    if ld < rows:
        raise ValueError("positions of different axes overlap")
    return positions.data_ptr(), i64, ld


def _rope(x, positions, plan, out, stream, inverse, name):
    if not isinstance(plan, RopePlan):
        raise TypeError("plan must be a RopePlan")
    if out is None and stream is None:
        return _done(_native().rope(x, positions, plan._at[inverse], name), "iso_rope")
    if stream is not None:
        with torch.cuda.stream(stream):
            return _rope(x, positions, plan, out, None, inverse, name)
    cfg = plan._cfg[inverse]
    dx = _mat(x, name)
    ptr, i64, ld = _positions(positions, dx.rows, plan.axes)
    s = _here(x, positions, out)
    if out is None:
        out, do = _new(dx.rows, dx.cols, x.dtype, x.device)
    else:
        do = _mat(out, "out")
    check(lib().iso_rope(_byref(dx), ptr, i64, ld, _byref(cfg), _byref(do), s), "iso_rope")
    return out


def rope(x: torch.Tensor, positions: torch.Tensor, plan: RopePlan, out: Optional[torch.Tensor] = None,
         stream=None) -> torch.Tensor:
    """x, heads of plan.head_dim side by side, turned by its rows' positions
    (iso_rope): int32 or int64 [axes, rows], or [rows] for one axis.  ``out`` may
    be x."""
    return _rope(x, positions, plan, out, stream, 0, "x")


def rope_grad(dy: torch.Tensor, positions: torch.Tensor, plan: RopePlan, out: Optional[torch.Tensor] = None,
              stream=None) -> torch.Tensor:
    """The gradient of rope's input: dy turned back (iso_rope with inverse)."""
    return _rope(dy, positions, plan, out, stream, 1, "dy")


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def _ends(t: Optional[torch.Tensor], name: str):
    if t is None:
        return None, 0
    if not isinstance(t, torch.Tensor) or t.dtype != torch.int32 or t.dim() != 1 or t.numel() < 2:
        raise TypeError(f"{name} must be a 1-D int32 tensor of the sequences' offsets and their end")
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA tensor")
    return t.data_ptr(), t.numel() - 1


def _attn_cfg(q: IsoMat, heads, kv_heads, scale, causal, window, seqs, kv_seqs, zero_rest=False) -> IsoAttnCfg:
    heads = int(heads)
    kv_heads = heads if kv_heads is None else int(kv_heads)
    if heads < 1 or kv_heads < 1 or heads % kv_heads:
        raise ValueError(f"{heads} query heads do not share {kv_heads} key heads evenly")
    if q.cols % heads or not q.cols:
        raise ValueError(f"{q.cols} columns are not {heads} heads")
    window = int(window or 0)
    if window < 0 or (window and not causal):
        raise ValueError("window must not be negative, and needs causal")
    (qe, n), (ke, nk) = _ends(seqs, "seqs"), _ends(kv_seqs, "kv_seqs")
    if ke is not None and nk != n:
        raise ValueError(f"kv_seqs holds {nk} sequences, seqs {n}")
    dim = q.cols // heads
    scale = dim ** -0.5 if scale is None else float(scale)
    if not (scale > 0 and math.isfinite(scale)):
        raise ValueError("scale must be positive and finite")
    return IsoAttnCfg(heads, kv_heads, dim, int(bool(causal)), min(window, 1 << 40), scale, n, qe, ke,
                      int(zero_rest), 0)


def attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, heads: int, kv_heads: Optional[int] = None,
         scale: Optional[float] = None, causal=True, window: int = 0, seqs: Optional[torch.Tensor] = None,
         kv_seqs: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
         lse: Optional[torch.Tensor] = None, workspace: Optional[Workspace] = None, status=False, stream=None):
    """(out, lse): attention of q's heads over k and v (iso_attn) and its
    log-sum-exp, float32 [heads, rows], which attn_grad takes.  ``kv_heads``
    (heads) key heads are shared by query heads in order; ``scale`` is
    head_dim^-0.5; ``window`` limits the keys a query sees (0: no limit).
    ``seqs`` holds the packed sequences' offsets and their end (int32 on the
    device), ``kv_seqs`` the keys' where they differ: queries stand at the end of
    their sequence's keys.  Rows of no sequence are zero in tensors that the call
    allocates; it does not write them where both out and lse are given.  With
    status=True the device status comes third."""
    if out is None and lse is None and workspace is None and stream is None and not status:
        return _done(_native().attn(q, k, v, heads, heads if kv_heads is None else kv_heads, scale, bool(causal), window or 0,
                                    seqs, kv_seqs), "iso_attn")
    if stream is not None:
        with torch.cuda.stream(stream):
            return attn(q, k, v, heads, kv_heads, scale, causal, window, seqs, kv_seqs, out, lse, workspace, status)
    dq, dk, dv = _mat(q, "q"), _mat(k, "k"), _mat(v, "v")
    cfg = _attn_cfg(dq, heads, kv_heads, scale, causal, window, seqs, kv_seqs, out is None or lse is None)
    s = _here(q, k, v, seqs, kv_seqs, out, lse)
    if out is None:
        out, do = _new(dq.rows, dq.cols, q.dtype, q.device)
    else:
        do = _mat(out, "out")
    if lse is None:
        lse = torch.empty((cfg.heads, dq.rows), dtype=torch.float32, device=q.device)
    lptr = _vector(lse, "lse", torch.float32, (cfg.heads, dq.rows))
    ws, st, L, nb = _scratch(workspace, q.device), _status(status, q.device), lib(), ctypes.c_size_t(0)
    check(L.iso_attn_workspace_size(_byref(dq), _byref(dk), _byref(cfg), _byref(nb)), "iso_attn")
    check(L.iso_attn(_byref(dq), _byref(dk), _byref(dv), _byref(cfg), _byref(do), lptr, *ws.get(nb.value), _ptr(st), s),
          "iso_attn")
    return (out, lse, st) if status else (out, lse)


def attn_grad(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
              lse: torch.Tensor, heads: int, kv_heads: Optional[int] = None, scale: Optional[float] = None,
              causal=True, window: int = 0, seqs: Optional[torch.Tensor] = None,
              kv_seqs: Optional[torch.Tensor] = None, grads: Optional[Tuple] = None,
              workspace: Optional[Workspace] = None, status=False, stream=None):
    """(dq, dk, dv) from the gradient of attn's out, its inputs, out and lse, with
    attn's other arguments (iso_attn_grad).  ``grads`` gives the tensors to write,
    possibly column ranges of one buffer; their rows of no sequence are not
    written (those of tensors that the call allocates are zero).  The same inputs
    give the same bits.  With status=True the device status comes fourth."""
    if grads is None and workspace is None and stream is None and not status:
        return _done(_native().attn_grad(dout, q, k, v, out, lse, heads, heads if kv_heads is None else kv_heads, scale,
                                         bool(causal), window or 0, seqs, kv_seqs), "iso_attn_grad")
    if stream is not None:
        with torch.cuda.stream(stream):
            return attn_grad(dout, q, k, v, out, lse, heads, kv_heads, scale, causal, window, seqs, kv_seqs, grads,
                             workspace, status)
    mq, mk, mv, mo, md = _mat(q, "q"), _mat(k, "k"), _mat(v, "v"), _mat(out, "out"), _mat(dout, "dout")
    cfg = _attn_cfg(mq, heads, kv_heads, scale, causal, window, seqs, kv_seqs, grads is None)
    lptr = _vector(lse, "lse", torch.float32, (cfg.heads, mq.rows))
    s = _here(q, k, v, out, dout, lse, seqs, kv_seqs)
    if grads is None:
        made = [_new(m.rows, m.cols, t.dtype, t.device) for m, t in ((mq, q), (mk, k), (mv, v))]
    else:
        if len(grads) != 3:
            raise ValueError("grads needs dq, dk and dv")
        made = [(t, _mat(t, n)) for t, n in zip(grads, ("dq", "dk", "dv"))]
        _here(q, *grads)
    (dq, a), (dk, b), (dv, c) = made
    ws, st, L, nb = _scratch(workspace, q.device), _status(status, q.device), lib(), ctypes.c_size_t(0)
    check(L.iso_attn_grad_workspace_size(_byref(mq), _byref(mk), _byref(cfg), _byref(nb)), "iso_attn_grad")
    check(L.iso_attn_grad(_byref(md), _byref(mq), _byref(mk), _byref(mv), _byref(mo), lptr, _byref(cfg), _byref(a),
                          _byref(b), _byref(c), *ws.get(nb.value), _ptr(st), s), "iso_attn_grad")
    return (dq, dk, dv, st) if status else (dq, dk, dv)


# ---------------------------------------------------------------------------
# distillation
# ---------------------------------------------------------------------------
def _tau(temperature) -> float:
    tau = float(temperature)
    if not (tau > 0 and math.isfinite(tau)):
        raise ValueError("temperature must be positive and finite")
    return tau


def _top(ids: torch.Tensor, teacher: IsoMat):
    i64 = _integers(ids, "ids")
    if tuple(ids.shape) != (teacher.rows, teacher.cols):
        raise ValueError(f"ids must have the teacher's shape {(teacher.rows, teacher.cols)}, has {tuple(ids.shape)}")
    if not ids.is_contiguous():
        raise ValueError("ids must be contiguous")
    return ids.data_ptr(), i64


def distill(logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, temperature=1.0,
            dloss: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, status=False, stream=None):
    """(loss, lse), float32 per row: the divergence of softmax(logits / tau) from
    the teacher's distribution over its top entries (iso_distill), ``ids`` and
    ``teacher`` [rows, K] its vocabulary ids (-1: unused slot) and logits.  With
    ``dloss`` (float32 per row) also the gradient of the logits, third, read in
    the same pass; into ``out``, which may be the logits.  With status=True the
    device status comes last."""
    if out is None and stream is None and not status:
        return _done(_native().distill(logits, ids, teacher, _tau(temperature), dloss), "iso_distill")
    if stream is not None:
        with torch.cuda.stream(stream):
            return distill(logits, ids, teacher, temperature, dloss, out, status)
    dz, dt = _mat(logits, "logits"), _mat(teacher, "teacher")
    ptr, i64 = _top(ids, dt)
    s = _here(logits, ids, teacher, dloss, out)
    loss, lse = torch.empty((2, dz.rows), dtype=torch.float32, device=logits.device).unbind(0)
    do = dptr = None
    if dloss is not None:
        dptr = _vector(dloss, "dloss", torch.float32, (dz.rows,))
        if out is None:
            out, do = _new(dz.rows, dz.cols, logits.dtype, logits.device)
        else:
            do = _mat(out, "out")
    elif out is not None:
        raise ValueError("out (the gradient) needs dloss")
    st = _status(status, logits.device)
    check(lib().iso_distill(_byref(dz), ptr, i64, _byref(dt), _tau(temperature), loss.data_ptr(), lse.data_ptr(), dptr,
                            None if do is None else _byref(do), _ptr(st), s), "iso_distill")
    return (loss, lse) + (() if do is None else (out,)) + ((st,) if status else ())


def distill_grad(dloss: torch.Tensor, logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor,
                 lse: torch.Tensor, temperature=1.0, out: Optional[torch.Tensor] = None, status=False, stream=None):
    """The gradient of distill's logits from that of its loss and its lse
    (iso_distill_grad); ``out`` may be the logits."""
    if out is None and stream is None and not status:
        return _done(_native().distill_grad(dloss, logits, ids, teacher, lse, _tau(temperature)), "iso_distill_grad")
    if stream is not None:
        with torch.cuda.stream(stream):
            return distill_grad(dloss, logits, ids, teacher, lse, temperature, out, status)
    dz, dt = _mat(logits, "logits"), _mat(teacher, "teacher")
    ptr, i64 = _top(ids, dt)
    dptr = _vector(dloss, "dloss", torch.float32, (dz.rows,))
    lptr = _vector(lse, "lse", torch.float32, (dz.rows,))
    s = _here(logits, ids, teacher, dloss, lse, out)
    if out is None:
        out, do = _new(dz.rows, dz.cols, logits.dtype, logits.device)
    else:
        do = _mat(out, "out")
    st = _status(status, logits.device)
    check(lib().iso_distill_grad(dptr, _byref(dz), ptr, i64, _byref(dt), _tau(temperature), lptr, _byref(do), _ptr(st),
                                 s), "iso_distill_grad")
    return (out, st) if status else out
