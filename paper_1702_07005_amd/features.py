"""Operators of learned features: table lookup, layer norm, their gradients, and gradient clipping.

They serve models whose coordinates are rows of a learned table instead of one-hot columns: ids are
looked up, the vectors normalised, a linear read-out is fitted on them by ``scd.Solver``, and the table is
trained by the read-out's gradient.  Every step runs in the HIP kernels of ``libscd.so``; this module
marshals arguments (``include/scd.h`` documents the calls) and allocates outputs and scratch from torch's
caching allocator, so the calls enqueue on a stream, never synchronise, and can be captured in graphs.

Matrices may be views with any row stride, but their last dimension has unit stride.  Work is enqueued on
the current stream, or on ``stream`` (a torch stream or a raw handle), with which the caller orders the
inputs; outputs that the call allocates then belong to that stream.

    x = features.embed(ids, table, scale=table.shape[1] ** 0.5)
    y, mean, rstd = features.layer_norm(x, weight, bias)
    dx, dw, db = features.layer_norm_grad(dy, x, mean, rstd, weight)
    dtable = features.embed_grad(ids, dx, table.shape[0], scale=table.shape[1] ** 0.5)
    norm = features.clip_grads([dtable, dw, db], 1.0)
"""
from __future__ import annotations

import contextlib
import ctypes

import torch

from .scd import _check, lib

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_TOKENS = {torch.int32: 3, torch.int64: 4}


class _Span(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("n", ctypes.c_int64), ("src_type", ctypes.c_int32),
                ("dst_type", ctypes.c_int32)]


def _on(device, stream):
    """A context in which the device and the stream are current (so that allocations belong to them), and
    the raw stream."""
    index = device.index
    if stream is None:
        raw = torch.cuda.current_stream(index).cuda_stream
        if index == torch.cuda.current_device():
            return contextlib.nullcontext(), raw
        return torch.cuda.device(index), raw
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    if stream.device != device:
        raise ValueError(f"the stream is on {stream.device}, the tensors on {device}")
    return torch.cuda.stream(stream), stream.cuda_stream


def _matrix(t, what, dtypes=_TYPES, device=None):
    """Checks a tensor of at least one dimension; returns it as rows (n, dim, row stride)."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dim() >= 1 and t.dtype in dtypes):
        raise ValueError(f"{what} must be a CUDA tensor of {', '.join(str(d)[6:] for d in dtypes)} with at least one dimension")
    if device is not None and t.device != device:
        raise ValueError(f"{what} is on {t.device}, other tensors on {device}")
    if t.dim() != 2:
        try:
            t = t.view(-1, t.shape[-1]) if t.shape[-1] else t.view(t.numel(), 0)
        except RuntimeError:
            raise ValueError(f"{what}: its leading dimensions must have one stride together") from None
    n, dim = t.shape
    if dim > 1 and t.stride(1) != 1:
        raise ValueError(f"{what}: its last dimension must have unit stride")
    return n, dim, t.stride(0) if n > 1 else dim


def _vector(t, what, dtype, n, device):
    if not (isinstance(t, torch.Tensor) and t.device == device and t.dtype == dtype and t.is_contiguous() and t.numel() == n):
        raise ValueError(f"{what} must be a contiguous {dtype} tensor with {n} elements on {device}")
    return t.data_ptr()


def _result(out, shape, dtype, device, what="out"):
    """`out` checked, or a new tensor; and its row stride."""
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=device)
        return out, shape[-1]
    if tuple(out.shape) != tuple(shape):
        raise ValueError(f"{what} must have the shape {tuple(shape)}")
    stride = _matrix(out, what, device=device)[2]
    if dtype is not None and out.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}")
    return out, stride


def embed(tokens, table, scale=1.0, out=None, dtype=None, stream=None):
    """``out[..., :] = scale * table[tokens[...], :]``; a negative token (a padded place) gives zeros, one of
    at least ``table.shape[0]`` NaN.

    ``tokens``: contiguous int32 or int64, any shape; ``table``: [rows, dim] of float32, bfloat16 or float16;
    ``dtype``: of the output (the table's by default)."""
    rows, dim, tstride = _matrix(table, "table")
    if table.dim() != 2:
        raise ValueError("table must have two dimensions")
    device = table.device
    if not (isinstance(tokens, torch.Tensor) and tokens.device == device and tokens.dtype in _TOKENS and tokens.is_contiguous()):
        raise ValueError("tokens must be a contiguous int32 or int64 tensor on the table's device")
    dtype = dtype if dtype is not None else out.dtype if out is not None else table.dtype
    if dtype not in _TYPES:
        raise ValueError("dtype must be float32, bfloat16 or float16")
    context, raw = _on(device, stream)
    with context:
        out, ostride = _result(out, (*tokens.shape, dim), dtype, device)
        _check(lib.scd_embed(tokens.data_ptr(), _TOKENS[tokens.dtype], tokens.numel(), table.data_ptr(), _TYPES[table.dtype],
                             tstride, rows, dim, scale, out.data_ptr(), _TYPES[dtype], ostride, raw))
    return out


def embed_grad(tokens, grad, rows, scale=1.0, out=None, accumulate=False, dtype=None, stream=None):
    """The gradient of ``embed`` with respect to its table: row v of [rows, dim] is ``scale`` times the sum of
    ``grad``'s rows whose token is v.  Tokens outside [0, rows) add to nothing.  ``accumulate`` adds to
    ``out`` instead of overwriting it.

    ``grad``: [*tokens.shape, dim]; ``dtype``: of the result (``grad``'s by default).  The result is
    bit-identical from call to call."""
    n, dim, gstride = _matrix(grad, "grad")
    device = grad.device
    if not (isinstance(tokens, torch.Tensor) and tokens.device == device and tokens.dtype in _TOKENS and tokens.is_contiguous()):
        raise ValueError("tokens must be a contiguous int32 or int64 tensor on the gradient's device")
    if grad.shape[:-1] != tokens.shape:
        raise ValueError(f"grad must have the shape {(*tokens.shape, 'dim')}")
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    dtype = dtype if dtype is not None else out.dtype if out is not None else grad.dtype
    if dtype not in _TYPES:
        raise ValueError("dtype must be float32, bfloat16 or float16")
    rows = int(rows)
    need = ctypes.c_int64()
    _check(lib.scd_embed_grad_workspace(n, rows, dim, ctypes.byref(need)))
    context, raw = _on(device, stream)
    with context:
        out, ostride = _result(out, (rows, dim), dtype, device)
        work = torch.empty(need.value, dtype=torch.uint8, device=device)
        _check(lib.scd_embed_grad(tokens.data_ptr(), _TOKENS[tokens.dtype], n, grad.data_ptr(), _TYPES[grad.dtype], gstride,
                                  rows, dim, scale, 1 if accumulate else 0, out.data_ptr(), _TYPES[dtype], ostride,
                                  work.data_ptr(), need.value, raw))
    return out


def layer_norm(x, weight=None, bias=None, eps=1e-5, out=None, stream=None):
    """``(x - mean) * rstd * weight + bias`` over the last dimension; returns it with ``mean`` and ``rstd``
    (float32, one for each row), which ``layer_norm_grad`` takes.

    ``weight`` and ``bias``: [dim], both of ``x``'s type or both float32, or None.  ``out`` may be ``x``."""
    n, dim, xstride = _matrix(x, "x")
    device = x.device
    param = weight.dtype if weight is not None else bias.dtype if bias is not None else x.dtype
    w = _vector(weight, "weight", param, dim, device) if weight is not None else None
    b = _vector(bias, "bias", param, dim, device) if bias is not None else None
    context, raw = _on(device, stream)
    with context:
        out, ostride = _result(out, x.shape, x.dtype, device)
        stats = torch.empty(2, *x.shape[:-1], dtype=torch.float32, device=device)
        mean, rstd = stats.unbind(0)
        _check(lib.scd_layer_norm(x.data_ptr(), _TYPES[x.dtype], xstride, n, dim, w, b, _TYPES.get(param, -1), eps,
                                  out.data_ptr(), ostride, mean.data_ptr(), rstd.data_ptr(), raw))
    return out, mean, rstd


def layer_norm_grad(grad, x, mean, rstd, weight=None, params=True, out=None, stream=None):
    """The gradients of ``layer_norm`` with respect to ``x``, ``weight`` and ``bias``, from the gradient of its
    output and the ``mean`` and ``rstd`` it returned.  Those of weight and bias have the weight's type (``x``'s
    where there is none) and are None with ``params=False``.  ``out`` (for ``x``'s) may be ``grad`` or ``x``."""
    n, dim, xstride = _matrix(x, "x")
    device = x.device
    gstride = _matrix(grad, "grad", device=device)[2]
    if grad.dtype != x.dtype or grad.shape != x.shape:
        raise ValueError("grad must have x's type and shape")
    m, r = _vector(mean, "mean", torch.float32, n, device), _vector(rstd, "rstd", torch.float32, n, device)
    param = weight.dtype if weight is not None else x.dtype
    w = _vector(weight, "weight", param, dim, device) if weight is not None else None
    dw = db = work = None
    need = ctypes.c_int64()
    if params:
        _check(lib.scd_layer_norm_grad_workspace(n, dim, ctypes.byref(need)))
    context, raw = _on(device, stream)
    with context:
        out, ostride = _result(out, x.shape, x.dtype, device)
        if params:
            dw, db = torch.empty(2, dim, dtype=param, device=device).unbind(0)
            work = torch.empty(need.value, dtype=torch.uint8, device=device)
        _check(lib.scd_layer_norm_grad(grad.data_ptr(), gstride, x.data_ptr(), xstride, _TYPES[x.dtype], m, r, n, dim, w,
                                       _TYPES.get(param, -1), out.data_ptr(), ostride, dw.data_ptr() if params else None,
                                       db.data_ptr() if params else None, work.data_ptr() if params else None, need.value, raw))
    return out, dw, db


_clip_bytes = ctypes.c_int64()
_check(lib.scd_clip_grads_workspace(ctypes.byref(_clip_bytes)))


def clip_grads(grads, max_norm, out=None, stream=None):
    """Scales the tensors of ``grads`` together so that their norm is at most ``max_norm``, in place or into the
    tensors of ``out`` (each of its gradient's type or float32).  Returns the norm before, a float32 tensor on
    the GPU, without waiting for it.

    The tensors are contiguous, of float32, bfloat16 or float16, and on one device."""
    grads = list(grads)
    outs = grads if out is None else list(out)
    if len(outs) != len(grads):
        raise ValueError("out must have as many tensors as grads")
    if not grads:
        raise ValueError("no gradients")
    return _clip(grads, outs, float(max_norm), stream)


def grad_norm(grads, stream=None):
    """The norm of all tensors of ``grads`` together: a float32 tensor on the GPU."""
    grads = list(grads)
    if not grads:
        raise ValueError("no gradients")
    return _clip(grads, None, float("inf"), stream)


def _clip(grads, outs, max_norm, stream):
    device = grads[0].device
    spans = (_Span * len(grads))()
    for i, g in enumerate(grads):
        o = outs[i] if outs is not None else None
        if not (g.is_cuda and g.device == device and g.dtype in _TYPES and g.is_contiguous()):
            raise ValueError(f"gradient {i} must be a contiguous float32, bfloat16 or float16 tensor on {device}")
        if o is not None and o is not g and not (o.device == device and o.shape == g.shape and o.is_contiguous()
                                                 and o.dtype in (g.dtype, torch.float32)):
            raise ValueError(f"output {i} must be contiguous, with its gradient's shape, and its type or float32")
        spans[i] = _Span(g.data_ptr(), o.data_ptr() if o is not None else None, g.numel(), _TYPES[g.dtype],
                         _TYPES[o.dtype] if o is not None else _TYPES[g.dtype])
    context, raw = _on(device, stream)
    with context:
        norm = torch.empty((), dtype=torch.float32, device=device)
        work = torch.empty(_clip_bytes.value, dtype=torch.uint8, device=device)
        _check(lib.scd_clip_grads(spans, len(grads), max_norm, norm.data_ptr(), work.data_ptr(), _clip_bytes.value, raw))
    return norm
