"""Operators at the end of a language model's step: residual add + root-mean-square norm, linear head + softmax
cross entropy, distillation from a teacher's top logits.

Argument marshalling for the entry points of ``include/bns.h``, in the manner of ``bns.py``: tensors are CUDA
tensors, work goes to the current CUDA stream, nothing falls back.  Row tensors are [..., columns] with dense rows;
leading dimensions are taken together, so a tensor is either contiguous or two-dimensional with a row stride.
Outputs are new dense tensors.  ``bns.BnsError`` carries the status of a refused call, ``TypeError`` stands for a tensor
of the wrong kind.
"""
from __future__ import annotations

import ctypes
from functools import lru_cache
from typing import Optional

import torch

from . import bns as _bns
from .bns import BF16, F32, BnsError

GROUP = 128              # columns of a scale in the grouped 8-bit form
FLAG_BAD_TARGET = 2      # bns.workspace_status of a head's workspace: a target at or above the vocabulary's size

_CODES = {torch.float32: F32, torch.bfloat16: BF16}
_INDEX = {torch.int32: 0, torch.int64: 1}


class _Rows(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int), ("columns", ctypes.c_int), ("dtype", ctypes.c_int)]


class _Head(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int), ("vocabulary", ctypes.c_int), ("width", ctypes.c_int), ("dtype", ctypes.c_int),
                ("x_stride", ctypes.c_int64), ("w_stride", ctypes.c_int64), ("target_is_int64", ctypes.c_int)]


class _Distillation(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int), ("vocabulary", ctypes.c_int), ("entries", ctypes.c_int), ("dtype", ctypes.c_int),
                ("stride", ctypes.c_int64), ("teacher_dtype", ctypes.c_int), ("index_is_int64", ctypes.c_int),
                ("temperature", ctypes.c_float)]


@lru_cache(maxsize=4096)
def _shape(kind, *fields):
    """(structure, reference to it) for these values; the library only reads it."""
    struct = kind(*fields)
    return struct, ctypes.byref(struct)


_lib = None


def _load():
    global _lib
    if _lib is None:
        lib = _bns.load()
        vp, sz, fl, i64, it = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float, ctypes.c_int64, ctypes.c_int
        rows, head, dist = (ctypes.POINTER(s) for s in (_Rows, _Head, _Distillation))
        for name, result, arguments in (
                ("bns_rms_norm_forward", it, [rows, vp, i64, vp, i64, vp, fl, vp, vp, vp, vp]),
                ("bns_rms_norm_forward_quantized", it, [rows, vp, i64, vp, i64, vp, fl, it, vp, vp, vp, vp, vp]),
                ("bns_rms_norm_workspace_bytes", sz, [rows]),
                ("bns_rms_norm_backward", it, [rows, vp, i64, vp, i64, vp, vp, vp, i64, vp, vp, vp, sz, vp]),
                ("bns_linear_cross_entropy_workspace_bytes", sz, [head, it]),
                ("bns_linear_cross_entropy_forward", it, [head, vp, vp, vp, vp, vp, vp, sz, vp]),
                ("bns_linear_cross_entropy_backward", it, [head, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
                ("bns_topk_distillation_forward", it, [dist, vp, vp, vp, vp, vp, vp]),
                ("bns_topk_distillation_backward", it, [dist, vp, vp, vp, vp, vp, vp, i64, vp]),
                ("bns_topk_distillation_step", it, [dist, vp, vp, vp, vp, vp, vp, i64, vp])):
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = result, arguments
        _lib = lib
    return _lib


# ----------------------------------------------------------------------------- tensors
def _matrix(t, name: str, like: Optional[torch.Tensor] = None):
    """(rows, columns, row stride) of a tensor whose rows are dense."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a CUDA tensor (this library has no CPU path)")
    if like is not None and (t.shape != like.shape or t.dtype != like.dtype or t.device != like.device):
        raise TypeError(f"{name} must match the other tensors in shape, dtype and device")
    n = t.dim()
    if n < 1 or t.shape[-1] == 0:
        raise TypeError(f"{name}: expected [..., columns] with at least one column")
    columns = t.shape[-1]
    if t.numel() // columns > 0x7FFFFFFF or columns > 0x7FFFFFFF:
        raise TypeError(f"{name}: more than 2^31 - 1 rows or columns")
    if t.is_contiguous():
        return t.numel() // columns, columns, columns
    if n == 2 and (t.stride(1) == 1 or columns == 1) and t.stride(0) >= columns:
        return t.shape[0], columns, t.stride(0)
    raise TypeError(f"{name}: rows must be dense, and more than two dimensions contiguous")


def _code(t: torch.Tensor) -> int:
    code = _CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported element type {t.dtype}")
    return code


def _vector(t, count: int, name: str, device, dtype=torch.float32) -> int:
    if (not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device != device or t.numel() != count
            or not t.is_contiguous()):
        raise TypeError(f"{name} must be a contiguous {dtype} tensor of {count} values on {device}")
    return t.data_ptr()


def _indices(t, shape, name: str, device):
    """(pointer, 1 for int64) of contiguous int32 or int64 indices."""
    if not isinstance(t, torch.Tensor) or t.device != device or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous index tensor of shape {tuple(shape)} on {device}")
    wide = _INDEX.get(t.dtype)
    if wide is None:
        raise TypeError(f"{name} must be int32 or int64")
    return t.data_ptr(), wide


def _stream(device) -> int:
    """The current stream, of the tensors' device: kernels are launched on the device that is current."""
    index = device.index
    if index != torch.cuda.current_device():
        raise TypeError(f"tensors are on {device}, the current device is cuda:{torch.cuda.current_device()}")
    return torch._C._cuda_getCurrentRawStream(index)      # torch.cuda.current_stream() builds a Stream object first: 3 us


def _check(status: int, what: str) -> None:
    if status != 0:
        raise BnsError(status, what)


def _like(t, dtype=None):
    """A new dense tensor of t's shape."""
    if t.is_contiguous():
        return torch.empty_like(t, dtype=dtype)
    return torch.empty(t.shape, dtype=dtype or t.dtype, device=t.device)


def _vector_of(t):
    """A new fp32 tensor with a value for each row of t."""
    return t.new_empty(t.shape[:-1], dtype=torch.float32)


def _scratch(workspace, need: int, device):
    if workspace is None:
        return torch.empty(need, dtype=torch.uint8, device=device)
    if workspace.device != device or not workspace.is_contiguous():
        raise TypeError(f"workspace must be a contiguous tensor on {device}")
    return workspace


# ----------------------------------------------------------------------------- root-mean-square norm
def _norm_inputs(x, residual, weight):
    rows, columns, stride = _matrix(x, "x")
    residual_stride, residual_at = columns, None
    if residual is not None:
        residual_stride = _matrix(residual, "residual", x)[2]
        residual_at = residual.data_ptr()
    shape = _shape(_Rows, rows, columns, _code(x))[1]
    return shape, x.data_ptr(), stride, residual_at, residual_stride, _vector(weight, columns, "weight", x.device)


def rms_norm_forward(x, residual, weight, eps):
    """bns_rms_norm_forward: returns (y, h, rstd) with h = x + residual and y = h rstd weight.  ``residual`` may be
    None; h is then x itself.  weight and rstd are float32."""
    shape, xp, xs, rp, rs, wp = _norm_inputs(x, residual, weight)
    y = _like(x)
    h = x if residual is None else _like(x)
    rstd = _vector_of(x)
    _check(_load().bns_rms_norm_forward(shape, xp, xs, rp, rs, wp, float(eps), y.data_ptr(),
                                        None if residual is None else h.data_ptr(), rstd.data_ptr(), _stream(x.device)),
           "bns_rms_norm_forward")
    return y, h, rstd


def rms_norm_forward_fp8(x, residual, weight, eps, group=0):
    """bns_rms_norm_forward_quantized: returns (q, scales, h, rstd); q is float8_e4m3fn, y = q * scale.  ``group``: 0 for
    one scale a row (scales [..., 1]), 128 for one per 128 columns (scales [..., ceil(columns / 128)])."""
    shape, xp, xs, rp, rs, wp = _norm_inputs(x, residual, weight)
    groups = 1 if group == 0 else -(-x.shape[-1] // GROUP)
    q = _like(x, torch.float8_e4m3fn)
    scales = x.new_empty((*x.shape[:-1], groups), dtype=torch.float32)
    h = x if residual is None else _like(x)
    rstd = _vector_of(x)
    _check(_load().bns_rms_norm_forward_quantized(shape, xp, xs, rp, rs, wp, float(eps), int(group),
                                                  q.data_ptr(), scales.data_ptr(),
                                                  None if residual is None else h.data_ptr(), rstd.data_ptr(),
                                                  _stream(x.device)), "bns_rms_norm_forward_quantized")
    return q, scales, h, rstd


def rms_norm_backward(dy, h, weight, rstd, dh=None, workspace=None):
    """bns_rms_norm_backward: returns (dx, dweight).  ``dh`` is the gradient that reaches h along the residual path; dx is
    the gradient of x and of the residual alike."""
    rows, columns, h_stride = _matrix(h, "h")
    dy_stride = _matrix(dy, "dy", h)[2]
    dh_stride, dh_at = columns, None
    if dh is not None:
        dh_stride, dh_at = _matrix(dh, "dh", h)[2], dh.data_ptr()
    device, lib = h.device, _load()
    weight_at = _vector(weight, columns, "weight", device)
    shape = _shape(_Rows, rows, columns, _code(h))[1]
    dx = _like(h)
    dweight = torch.empty_like(weight)
    workspace = _scratch(workspace, lib.bns_rms_norm_workspace_bytes(shape), device)
    _check(lib.bns_rms_norm_backward(shape, dy.data_ptr(), dy_stride, h.data_ptr(), h_stride,
                                     weight_at, _vector(rstd, rows, "rstd", device), dh_at,
                                     dh_stride, dx.data_ptr(), dweight.data_ptr(), workspace.data_ptr(), workspace.nbytes,
                                     _stream(device)), "bns_rms_norm_backward")
    return dx, dweight


# ----------------------------------------------------------------------------- linear head + cross entropy
def _head_inputs(x, w, target):
    rows, width, x_stride = _matrix(x, "x")
    vocabulary, w_width, w_stride = _matrix(w, "w")
    if w.dim() != 2 or w_width != width or w.dtype != x.dtype or w.device != x.device:
        raise TypeError("w must be [vocabulary, width] with the width, dtype and device of x")
    at, wide = _indices(target, x.shape[:-1], "target", x.device)
    return (*_shape(_Head, rows, vocabulary, width, _code(x), x_stride, w_stride, wide), at)


def linear_cross_entropy_workspace_bytes(x, w, target, backward=False) -> int:
    _, shape, _ = _head_inputs(x, w, target)
    need = _load().bns_linear_cross_entropy_workspace_bytes(shape, 1 if backward else 0)
    if need == 0:
        raise BnsError(-2, "bns_linear_cross_entropy_workspace_bytes")
    return int(need)


def linear_cross_entropy_forward(x, w, target, workspace=None):
    """bns_linear_cross_entropy_forward: returns (loss, lse), float32 of target's shape.  Rows whose target is negative
    are left out: their loss is 0.  The caller takes the mean, or whatever it wants, of the losses."""
    _, shape, at = _head_inputs(x, w, target)
    device, lib = x.device, _load()
    loss, lse = torch.empty_like(target, dtype=torch.float32), torch.empty_like(target, dtype=torch.float32)
    workspace = _scratch(workspace, lib.bns_linear_cross_entropy_workspace_bytes(shape, 0), device)
    _check(lib.bns_linear_cross_entropy_forward(shape, x.data_ptr(), w.data_ptr(), at, loss.data_ptr(),
                                                lse.data_ptr(), workspace.data_ptr(), workspace.nbytes, _stream(device)),
           "bns_linear_cross_entropy_forward")
    return loss, lse


def linear_cross_entropy_backward(x, w, target, lse, dloss, workspace=None):
    """bns_linear_cross_entropy_backward: returns (dx, dw); dloss is the gradient of every row's loss, float32."""
    fields, shape, at = _head_inputs(x, w, target)
    device, lib = x.device, _load()
    dx, dw = _like(x), _like(w)
    workspace = _scratch(workspace, lib.bns_linear_cross_entropy_workspace_bytes(shape, 1), device)
    _check(lib.bns_linear_cross_entropy_backward(shape, x.data_ptr(), w.data_ptr(), at,
                                                 _vector(lse, fields.rows, "lse", device),
                                                 _vector(dloss, fields.rows, "dloss", device), dx.data_ptr(), dw.data_ptr(),
                                                 workspace.data_ptr(), workspace.nbytes, _stream(device)),
           "bns_linear_cross_entropy_backward")
    return dx, dw


# ----------------------------------------------------------------------------- distillation
def _distillation_inputs(logits, teacher, index, temperature):
    rows, vocabulary, stride = _matrix(logits, "logits")
    if (not isinstance(teacher, torch.Tensor) or teacher.device != logits.device or teacher.dim() != logits.dim()
            or teacher.shape[:-1] != logits.shape[:-1] or not teacher.is_contiguous()):
        raise TypeError("teacher must be a contiguous tensor [..., entries] next to the logits")
    at, wide = _indices(index, teacher.shape, "index", logits.device)
    return (*_shape(_Distillation, rows, vocabulary, teacher.shape[-1], _code(logits), stride, _code(teacher), wide,
                    float(temperature)), at)


def topk_distillation_forward(logits, teacher, index, temperature=1.0):
    """bns_topk_distillation_forward: returns (loss, lse), float32 per row.  ``teacher`` holds the teacher's logits at the
    places ``index``; a negative index is no entry."""
    _, shape, at = _distillation_inputs(logits, teacher, index, temperature)
    loss, lse = _vector_of(logits), _vector_of(logits)
    _check(_load().bns_topk_distillation_forward(shape, logits.data_ptr(), teacher.data_ptr(), at,
                                                 loss.data_ptr(), lse.data_ptr(), _stream(logits.device)),
           "bns_topk_distillation_forward")
    return loss, lse


def topk_distillation_backward(logits, teacher, index, lse, dloss, temperature=1.0):
    """bns_topk_distillation_backward: the gradient of the logits; lse is what the forward call returned, dloss the gradient
    of every row's loss."""
    fields, shape, at = _distillation_inputs(logits, teacher, index, temperature)
    device = logits.device
    dlogits = _like(logits)
    _check(_load().bns_topk_distillation_backward(shape, logits.data_ptr(), teacher.data_ptr(), at,
                                                  _vector(lse, fields.rows, "lse", device),
                                                  _vector(dloss, fields.rows, "dloss", device), dlogits.data_ptr(),
                                                  fields.vocabulary, _stream(device)), "bns_topk_distillation_backward")
    return dlogits


def topk_distillation_step(logits, teacher, index, dloss, temperature=1.0):
    """bns_topk_distillation_step: returns (loss, dlogits) in one launch, for a dloss that is known beforehand (a mean over
    the rows, say)."""
    fields, shape, at = _distillation_inputs(logits, teacher, index, temperature)
    device = logits.device
    loss = torch.empty_like(dloss) if dloss.shape == logits.shape[:-1] else _vector_of(logits)
    dlogits = _like(logits)
    _check(_load().bns_topk_distillation_step(shape, logits.data_ptr(), teacher.data_ptr(), at,
                                              _vector(dloss, fields.rows, "dloss", device), loss.data_ptr(),
                                              dlogits.data_ptr(), fields.vocabulary, _stream(device)),
           "bns_topk_distillation_step")
    return loss, dlogits
