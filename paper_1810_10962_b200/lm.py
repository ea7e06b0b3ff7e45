"""Operators of a language model's step: residual add + root-mean-square norm, linear head + softmax cross entropy,
distillation from a teacher's top logits, log probabilities of given tokens, norm + rotation of queries' and keys' heads,
the norm over all gradients and clipping by it.

Argument marshalling for the entry points of ``include/bns.h``, in the manner of ``bns.py``: tensors are CUDA
tensors, work goes to the current CUDA stream, nothing falls back.  Row tensors are [..., columns] with dense rows;
leading dimensions are taken together, so a tensor is either contiguous or two-dimensional with a row stride.
Outputs are new dense tensors, but for clipped gradients.  ``bns.BnsError`` carries the status of a refused call, ``TypeError`` stands for a tensor
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


class _LogProbs(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int), ("vocabulary", ctypes.c_int), ("entries", ctypes.c_int), ("dtype", ctypes.c_int),
                ("stride", ctypes.c_int64), ("token_is_int64", ctypes.c_int), ("temperature", ctypes.c_float)]


class _HeadNorm(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int) for name in ("batch", "length", "q_heads", "k_heads", "head_dim", "rotary", "dtype")] + [
        (name, ctypes.c_int64) for name in ("q_batch", "q_position", "q_head", "k_batch", "k_position", "k_head")] + [
        ("positions", ctypes.c_int), ("position_is_int64", ctypes.c_int), ("interleaved", ctypes.c_int), ("eps", ctypes.c_float)]


class _Gradients(ctypes.Structure):
    _fields_ = [("count", ctypes.c_int), ("data", ctypes.c_void_p), ("out", ctypes.c_void_p), ("elements", ctypes.c_void_p),
                ("dtype", ctypes.c_void_p)]


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
        rows, head, dist, logp, turn, grads = (ctypes.POINTER(s) for s in (_Rows, _Head, _Distillation, _LogProbs, _HeadNorm,
                                                                           _Gradients))
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
                ("bns_topk_distillation_step", it, [dist, vp, vp, vp, vp, vp, vp, i64, vp]),
                ("bns_token_log_probs_forward", it, [logp, *[vp] * 8]),
                ("bns_token_log_probs_backward", it, [logp, *[vp] * 7, i64, vp]),
                ("bns_head_norm_rotary_forward", it, [turn, *[vp] * 10]),
                ("bns_head_norm_rotary_workspace_bytes", sz, [turn]),
                ("bns_head_norm_rotary_backward", it, [turn, *[vp] * 14, sz, vp]),
                ("bns_gradient_norm_workspace_bytes", sz, [grads]),
                ("bns_gradient_norm", it, [grads, vp, vp, sz, vp]),
                ("bns_clip_gradients", it, [grads, fl, vp, vp, sz, vp])):
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


# ----------------------------------------------------------------------------- log probabilities of given tokens
def _log_probs_inputs(logits, token, temperature, entries=0):
    rows, vocabulary, stride = _matrix(logits, "logits")
    at, wide = _indices(token, logits.shape[:-1], "token", logits.device)
    return (*_shape(_LogProbs, rows, vocabulary, entries, _code(logits), stride, wide, float(temperature)), at)


def _vectors_of(token):
    """Three new fp32 tensors of token's shape (empty_like takes half as long as new_empty: 1 us)."""
    first = torch.empty_like(token, dtype=torch.float32)
    return first, torch.empty_like(first), torch.empty_like(first)


def _dense_like(t):
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def token_log_probs_forward(logits, token, temperature=1.0):
    """bns_token_log_probs_forward without alternatives: returns (logprob, entropy, lse), float32 per row: the log probability
    of ``token`` under softmax(logits / temperature), 0 where it is negative, and the distribution's entropy."""
    _, shape, at = _log_probs_inputs(logits, token, temperature)
    logprob, entropy, lse = _vectors_of(token)
    _check(_load().bns_token_log_probs_forward(shape, logits.data_ptr(), at, logprob.data_ptr(), entropy.data_ptr(),
                                               lse.data_ptr(), None, None, _stream(logits.device)),
           "bns_token_log_probs_forward")
    return logprob, entropy, lse


def token_log_probs_forward_top(logits, token, entries, temperature=1.0):
    """bns_token_log_probs_forward with alternatives: returns (logprob, entropy, lse, top_logprob, top_index); the last two
    are [..., entries], float32 and int32, the largest logit first and the lowest place first among equals.  1 to 64
    entries."""
    if entries < 1:
        raise ValueError("entries must be at least 1")
    _, shape, at = _log_probs_inputs(logits, token, temperature, int(entries))
    logprob, entropy, lse = _vectors_of(token)
    top = logits.new_empty((*token.shape, entries), dtype=torch.float32)
    index = torch.empty_like(top, dtype=torch.int32)
    _check(_load().bns_token_log_probs_forward(shape, logits.data_ptr(), at, logprob.data_ptr(), entropy.data_ptr(),
                                               lse.data_ptr(), top.data_ptr(), index.data_ptr(), _stream(logits.device)),
           "bns_token_log_probs_forward")
    return logprob, entropy, lse, top, index


def token_log_probs_backward(logits, token, lse, entropy, dlogprob, dentropy=None, temperature=1.0):
    """bns_token_log_probs_backward: the gradient of the logits; lse and entropy are what the forward call returned,
    dlogprob and dentropy the gradients of every row's outputs.  Without dentropy the entropy may be None."""
    fields, shape, at = _log_probs_inputs(logits, token, temperature)
    device, rows = logits.device, fields.rows
    entropy_at = dentropy_at = None
    if dentropy is not None:
        entropy_at, dentropy_at = _vector(entropy, rows, "entropy", device), _vector(dentropy, rows, "dentropy", device)
    dlogits = _like(logits)
    _check(_load().bns_token_log_probs_backward(shape, logits.data_ptr(), at, _vector(lse, rows, "lse", device), entropy_at,
                                                _vector(dlogprob, rows, "dlogprob", device), dentropy_at, dlogits.data_ptr(),
                                                fields.vocabulary, _stream(device)), "bns_token_log_probs_backward")
    return dlogits


# ----------------------------------------------------------------------------- norm + rotation of heads
def _heads(t, name: str):
    """(batch, length, heads, head_dim, strides) of [length, heads, head_dim] or [batch, length, heads, head_dim]."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a CUDA tensor (this library has no CPU path)")
    shape, strides = t.shape, t.stride()
    n = len(shape)
    if n not in (3, 4):
        raise TypeError(f"{name}: expected [length, heads, head_dim] or [batch, length, heads, head_dim]")
    if strides[-1] != 1 and shape[-1] != 1:
        raise TypeError(f"{name}: heads must be dense")
    return (1, *shape, 0, *strides[:2]) if n == 3 else (*shape, *strides[:3])


def _head_norm_inputs(q, k, q_weight, k_weight, cos, sin, position, eps, interleaved):
    batch, length, heads, dim, *strides = _heads(q, "q")
    device, k_heads, k_strides, k_at, k_weight_at = q.device, 0, (0, 0, 0), None, None
    if k is not None:
        k_batch, k_length, k_heads, k_dim, *k_strides = _heads(k, "k")
        if (k_batch, k_length, k_dim) != (batch, length, dim) or k.dim() != q.dim() or k.dtype != q.dtype or k.device != device:
            raise TypeError("k must match q in positions, head_dim, dtype and device")
        k_at, k_weight_at = k.data_ptr(), _vector(k_weight, dim, "k_weight", device)
    if not isinstance(cos, torch.Tensor) or cos.dim() != 2:
        raise TypeError("cos must be [positions, rotary / 2]")
    positions, half = cos.shape
    at, wide = _indices(position, q.shape[:-2], "position", device)
    fields, shape = _shape(_HeadNorm, batch, length, heads, k_heads, dim, 2 * half, _code(q), *strides, *k_strides, positions,
                           wide, 1 if interleaved else 0, float(eps))
    return fields, shape, (q.data_ptr(), k_at, _vector(q_weight, dim, "q_weight", device), k_weight_at,
                   _vector(cos, positions * half, "cos", device), _vector(sin, positions * half, "sin", device), at)


def head_norm_rotary_forward(q, k, q_weight, k_weight, cos, sin, position, eps, interleaved=False):
    """bns_head_norm_rotary_forward: returns (q_out, k_out).  q and k are [length, heads, head_dim] or [batch, length, heads,
    head_dim], their heads dense, anything else strided (views of a packed projection); k and k_weight may be None.  cos
    and sin are float32 [positions, rotary / 2], position int32 or int64 in the shape of q's leading dimensions; a negative
    one is padding, whose outputs are zeros."""
    _, shape, arguments = _head_norm_inputs(q, k, q_weight, k_weight, cos, sin, position, eps, interleaved)
    q_out = _dense_like(q)
    k_out = None if k is None else _dense_like(k)
    _check(_load().bns_head_norm_rotary_forward(shape, *arguments, q_out.data_ptr(), None if k is None else k_out.data_ptr(),
                                                _stream(q.device)), "bns_head_norm_rotary_forward")
    return q_out, k_out


def _match(d, t, name: str) -> None:
    if (not isinstance(d, torch.Tensor) or d.shape != t.shape or d.dtype != t.dtype or d.device != t.device
            or not d.is_contiguous()):
        raise TypeError(f"{name} must be contiguous and match its input in shape, dtype and device")


def head_norm_rotary_backward(dq_out, dk_out, q, k, q_weight, k_weight, cos, sin, position, eps, interleaved=False,
                              workspace=None):
    """bns_head_norm_rotary_backward: returns (dq, dk, dq_weight, dk_weight) from the contiguous gradients of the outputs and
    the inputs of the forward call."""
    fields, shape, arguments = _head_norm_inputs(q, k, q_weight, k_weight, cos, sin, position, eps, interleaved)
    device, lib = q.device, _load()
    _match(dq_out, q, "dq_out")
    dq, dq_weight = _dense_like(q), torch.empty_like(q_weight)
    dk = dk_weight = dk_at = dk_out_at = dk_weight_at = None
    if k is not None:
        _match(dk_out, k, "dk_out")
        dk, dk_weight = _dense_like(k), torch.empty_like(k_weight)
        dk_at, dk_out_at, dk_weight_at = dk.data_ptr(), dk_out.data_ptr(), dk_weight.data_ptr()
    need = getattr(fields, "workspace_bytes", None)
    if need is None:
        need = fields.workspace_bytes = lib.bns_head_norm_rotary_workspace_bytes(shape)
    workspace = _scratch(workspace, need, device)
    _check(lib.bns_head_norm_rotary_backward(shape, dq_out.data_ptr(), dk_out_at, *arguments, dq.data_ptr(), dk_at,
                                             dq_weight.data_ptr(), dk_weight_at, workspace.data_ptr(), workspace.nbytes,
                                             _stream(device)), "bns_head_norm_rotary_backward")
    return dq, dk, dq_weight, dk_weight


# ----------------------------------------------------------------------------- norm over many gradients, clipping
def _dense(t) -> bool:
    """Whether the tensor's elements fill its span of memory, in any order of the dimensions."""
    if t.is_contiguous():
        return True
    expected = 1
    for stride, size in sorted(zip(t.stride(), t.shape)):
        if size != 1:
            if stride != expected:
                return False
            expected *= size
    return True


class GradientList:
    """Gradients whose norm is taken together, checked and laid out once for many steps.

    ``gradients``: dense tensors, float32 or bfloat16, in any mixture; ``out``: where clipped gradients go, tensors of the
    same shapes, types and strides, or None to clip in place.  The list keeps the tensors; their memory has to stay where it
    is."""

    def __init__(self, gradients, out=None):
        gradients = list(gradients)
        out = gradients if out is None else list(out)
        if len(out) != len(gradients):
            raise TypeError("out must have a tensor for each gradient")
        spans = []
        for i, (g, o) in enumerate(zip(gradients, out)):
            if not isinstance(g, torch.Tensor) or not g.is_cuda:
                raise TypeError(f"gradient {i}: expected a CUDA tensor (this library has no CPU path)")
            if g.device != gradients[0].device or not _dense(g):
                raise TypeError(f"gradient {i} must be dense and on the device of the first one")
            if o is not g and (not isinstance(o, torch.Tensor) or o.shape != g.shape or o.dtype != g.dtype
                               or o.device != g.device or o.stride() != g.stride()):
                raise TypeError(f"out {i} must match its gradient in shape, strides, dtype and device")
            _code(g)
            if g.numel():
                start, to = g.data_ptr(), o.data_ptr()
                if start != to:
                    spans.append((start, start + g.nbytes, False))
                spans.append((to, to + o.nbytes, True))
        self._overlap = False           # of an output with another one or a gradient: clipping would depend on the order
        read = written = 0
        for start, end, is_out in sorted(spans):
            self._overlap |= start < (max(read, written) if is_out else written)
            if is_out:
                written = max(written, end)
            else:
                read = max(read, end)
        n = len(gradients)
        self.gradients, self.out = gradients, out
        self._arrays = ((ctypes.c_void_p * n)(*(g.data_ptr() for g in gradients)),
                        (ctypes.c_void_p * n)(*(o.data_ptr() for o in out)),
                        (ctypes.c_int64 * n)(*(g.numel() for g in gradients)),
                        (ctypes.c_int * n)(*(_code(g) for g in gradients)))
        self._list = _Gradients(n, *(ctypes.addressof(a) for a in self._arrays))
        self._reference = ctypes.byref(self._list)
        self._device = gradients[0].device if n else torch.device("cuda", torch.cuda.current_device())
        need = _load().bns_gradient_norm_workspace_bytes(self._reference)
        # new tensors are made like these: half the time of torch.empty
        self._scratch = torch.empty(need, dtype=torch.uint8, device=self._device)
        self._norm = torch.empty((), dtype=torch.float32, device=self._device)

    def norm(self, workspace=None):
        """bns_gradient_norm: the norm over all elements of all gradients, a float32 scalar on the device."""
        stream = _stream(self._device)
        workspace = torch.empty_like(self._scratch) if workspace is None else _scratch(workspace, 0, self._device)
        norm = torch.empty_like(self._norm)
        _check(_load().bns_gradient_norm(self._reference, norm.data_ptr(), workspace.data_ptr(), workspace.nbytes, stream),
               "bns_gradient_norm")
        return norm

    def clip(self, max_norm, workspace=None):
        """bns_clip_gradients: writes the gradients, scaled down to ``max_norm`` where their norm is larger, to ``out``, and
        returns the norm that they had."""
        if self._overlap:
            raise TypeError("outputs overlap one another or another gradient")
        stream = _stream(self._device)
        workspace = torch.empty_like(self._scratch) if workspace is None else _scratch(workspace, 0, self._device)
        norm = torch.empty_like(self._norm)
        _check(_load().bns_clip_gradients(self._reference, float(max_norm), norm.data_ptr(), workspace.data_ptr(),
                                          workspace.nbytes, stream), "bns_clip_gradients")
        return norm


def gradient_norm(gradients):
    """The norm over all elements of the gradients (tensors, or a GradientList)."""
    return (gradients if isinstance(gradients, GradientList) else GradientList(gradients)).norm()


def clip_gradients(gradients, max_norm, out=None):
    """Clips the gradients (tensors, or a GradientList, which has its own ``out``) by their common norm, in place where
    ``out`` is None; returns the norm that they had.  Checking and laying out tensors takes some 2 us for each in every
    call; a GradientList has that done once."""
    if isinstance(gradients, GradientList):
        if out is not None:
            raise TypeError("a GradientList has its own out")
        return gradients.clip(max_norm)
    return GradientList(gradients, out).clip(max_norm)
