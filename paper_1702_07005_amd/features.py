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

import ctypes
import functools
from operator import attrgetter, eq

import torch

from .scd import _check, lib

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_TOKENS = {torch.int32: 3, torch.int64: 4}
_current_device = torch._C._cuda_getDevice
_current_stream = torch._C._cuda_getCurrentRawStream


def _other(device, stream):
    """None where the call's work belongs to the current stream and device; else a context that makes them so."""
    if stream is None:
        return None if device.index == _current_device() else torch.cuda.device(device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    if stream.device != device:
        raise ValueError(f"the stream is on {stream.device}, the tensors on {device}")
    return torch.cuda.stream(stream)


def _matrix(t, what, device=None):
    """A tensor of at least one dimension as rows: (rows, dim, row stride, type)."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{what} must be a tensor")
    kind, shape = _TYPES.get(t.dtype), t.shape
    if kind is None or not t.is_cuda or not shape:
        raise ValueError(f"{what} must be a CUDA tensor of float32, bfloat16 or float16 with at least one dimension")
    if device is not None and t.device != device:
        raise ValueError(f"{what} is on {t.device}, other tensors on {device}")
    dim = shape[-1]
    if t.is_contiguous():
        return t.numel() // dim if dim else 0, dim, dim, kind
    if len(shape) != 2:
        try:
            t = t.view(-1, dim)
        except RuntimeError:
            raise ValueError(f"{what}: its leading dimensions must have one stride together") from None
    n = t.shape[0]
    if dim > 1 and t.stride(1) != 1:
        raise ValueError(f"{what}: its last dimension must have unit stride")
    return n, dim, t.stride(0) if n > 1 else dim, kind


def _vector(t, what, dtype, n, device):
    if not (isinstance(t, torch.Tensor) and t.dtype == dtype and t.numel() == n and t.is_contiguous() and t.device == device):
        raise ValueError(f"{what} must be a contiguous {dtype} tensor with {n} elements on {device}")
    return t.data_ptr()


def _ids(tokens, device):
    kind = _TOKENS.get(tokens.dtype) if isinstance(tokens, torch.Tensor) else None
    if kind is None or tokens.device != device or not tokens.is_contiguous():
        raise ValueError(f"tokens must be a contiguous int32 or int64 tensor on {device}")
    return kind


def _result(out, shape, dtype, device):
    """The row stride of an output that the caller gave."""
    if not isinstance(out, torch.Tensor) or out.shape != shape or out.dtype != dtype:
        raise ValueError(f"out must be a {dtype} tensor of the shape {tuple(shape)}")
    return _matrix(out, "out", device)[2]


@functools.lru_cache(maxsize=1024)
def _scratch(call, *sizes):
    """The bytes of workspace that a call needs for its sizes."""
    need = ctypes.c_int64()
    _check(getattr(lib, call)(*sizes, ctypes.byref(need)))
    return need.value


def embed(tokens, table, scale=1.0, out=None, dtype=None, stream=None):
    """``out[..., :] = scale * table[tokens[...], :]``; a negative token (a padded place) gives zeros, one of
    at least ``table.shape[0]`` NaN.

    ``tokens``: contiguous int32 or int64, any shape; ``table``: [rows, dim] of float32, bfloat16 or float16;
    ``dtype``: of the output (the table's by default)."""
    rows, dim, tstride, kind = _matrix(table, "table")
    if table.dim() != 2:
        raise ValueError("table must have two dimensions")
    device = table.device
    ids = _ids(tokens, device)
    other = _other(device, stream)
    if other is not None:
        with other:
            return embed(tokens, table, scale, out, dtype)
    ostride = dim
    if out is not None:
        dtype = dtype or out.dtype
        ostride = _result(out, (*tokens.shape, dim), dtype, device)
    else:
        dtype = dtype or table.dtype
        if dtype not in _TYPES:
            raise ValueError("dtype must be float32, bfloat16 or float16")
        out = torch.empty((*tokens.shape, dim), dtype=dtype, device=device)
    _check(lib.scd_embed(tokens.data_ptr(), ids, tokens.numel(), table.data_ptr(), kind, tstride, table.shape[0], dim, scale,
                         out.data_ptr(), _TYPES[dtype], ostride, _current_stream(device.index)))
    return out


def embed_grad(tokens, grad, rows, scale=1.0, out=None, accumulate=False, dtype=None, stream=None):
    """The gradient of ``embed`` with respect to its table: row v of [rows, dim] is ``scale`` times the sum of
    ``grad``'s rows whose token is v.  Tokens outside [0, rows) add to nothing.  ``accumulate`` adds to
    ``out`` instead of overwriting it.

    ``grad``: [*tokens.shape, dim]; ``dtype``: of the result (``grad``'s by default).  The result is
    bit-identical from call to call."""
    n, dim, gstride, kind = _matrix(grad, "grad")
    device = grad.device
    ids = _ids(tokens, device)
    if grad.shape[:-1] != tokens.shape:
        raise ValueError(f"grad must have the shape {(*tokens.shape, 'dim')}")
    other = _other(device, stream)
    if other is not None:
        with other:
            return embed_grad(tokens, grad, rows, scale, out, accumulate, dtype)
    rows = int(rows)
    need = _scratch("scd_embed_grad_workspace", n, rows, dim)
    ostride = dim
    if out is not None:
        dtype = dtype or out.dtype
        ostride = _result(out, (rows, dim), dtype, device)
    elif accumulate:
        raise ValueError("accumulate needs out")
    else:
        dtype = dtype or grad.dtype
        if dtype not in _TYPES:
            raise ValueError("dtype must be float32, bfloat16 or float16")
        out = torch.empty((rows, dim), dtype=dtype, device=device)
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    _check(lib.scd_embed_grad(tokens.data_ptr(), ids, n, grad.data_ptr(), kind, gstride, rows, dim, scale, bool(accumulate),
                              out.data_ptr(), _TYPES[dtype], ostride, work.data_ptr() if need else None, need, _current_stream(device.index)))
    return out


def layer_norm(x, weight=None, bias=None, eps=1e-5, out=None, stream=None):
    """``(x - mean) * rstd * weight + bias`` over the last dimension; returns it with ``mean`` and ``rstd``
    (float32, one for each row), which ``layer_norm_grad`` takes.

    ``weight`` and ``bias``: [dim], both of ``x``'s type or both float32, or None.  ``out`` may be ``x``."""
    n, dim, xstride, kind = _matrix(x, "x")
    device = x.device
    param = weight.dtype if weight is not None else bias.dtype if bias is not None else x.dtype
    w = _vector(weight, "weight", param, dim, device) if weight is not None else None
    b = _vector(bias, "bias", param, dim, device) if bias is not None else None
    other = _other(device, stream)
    if other is not None:
        with other:
            return layer_norm(x, weight, bias, eps, out)
    shape, ostride = x.shape, dim
    if out is not None:
        ostride = _result(out, shape, x.dtype, device)
    else:
        out = torch.empty(shape, dtype=x.dtype, device=device)
    mean, rstd = torch.empty((2, *shape[:-1]), dtype=torch.float32, device=device).unbind()
    _check(lib.scd_layer_norm(x.data_ptr(), kind, xstride, n, dim, w, b, _TYPES.get(param, -1), eps, out.data_ptr(), ostride,
                              mean.data_ptr(), rstd.data_ptr(), _current_stream(device.index)))
    return out, mean, rstd


def layer_norm_grad(grad, x, mean, rstd, weight=None, params=True, out=None, stream=None):
    """The gradients of ``layer_norm`` with respect to ``x``, ``weight`` and ``bias``, from the gradient of its
    output and the ``mean`` and ``rstd`` it returned.  Those of weight and bias have the weight's type (``x``'s
    where there is none) and are None with ``params=False``.  ``out`` (for ``x``'s) may be ``grad`` or ``x``."""
    n, dim, xstride, kind = _matrix(x, "x")
    device, dtype = x.device, x.dtype
    gstride = _matrix(grad, "grad", device)[2]
    if grad.dtype != dtype or grad.shape != x.shape:
        raise ValueError("grad must have x's type and shape")
    m, r = _vector(mean, "mean", torch.float32, n, device), _vector(rstd, "rstd", torch.float32, n, device)
    param = weight.dtype if weight is not None else dtype
    w = _vector(weight, "weight", param, dim, device) if weight is not None else None
    other = _other(device, stream)
    if other is not None:
        with other:
            return layer_norm_grad(grad, x, mean, rstd, weight, params, out)
    ostride = dim
    if out is not None:
        ostride = _result(out, x.shape, dtype, device)
    else:
        out = torch.empty(x.shape, dtype=dtype, device=device)
    dw = db = pw = pb = work = None
    need = 0
    if params:
        need = _scratch("scd_layer_norm_grad_workspace", n, dim)
        dw, db = torch.empty((2, dim), dtype=param, device=device).unbind()
        pw, pb = dw.data_ptr(), db.data_ptr()
        if need:
            scratch = torch.empty(need, dtype=torch.uint8, device=device)
            work = scratch.data_ptr()
    _check(lib.scd_layer_norm_grad(grad.data_ptr(), gstride, x.data_ptr(), xstride, kind, m, r, n, dim, w, _TYPES.get(param, -1),
                                   out.data_ptr(), ostride, pw, pb, work, need, _current_stream(device.index)))
    return out, dw, db


def clip_grads(grads, max_norm, out=None, stream=None):
    """Scales the tensors of ``grads`` together so that their norm is at most ``max_norm``, in place or into the
    tensors of ``out`` (each of its gradient's type or float32).  Returns the norm before, a float32 tensor on
    the GPU, without waiting for it.

    The tensors are contiguous, of float32, bfloat16 or float16, and on one device."""
    return _clip(grads, grads if out is None else out, max_norm, stream)


def grad_norm(grads, stream=None):
    """The norm of all tensors of ``grads`` together: a float32 tensor on the GPU."""
    return _clip(grads, None, float("inf"), stream)


_Tensor = torch.Tensor
_dtype = attrgetter("dtype")
_shape = attrgetter("shape")


def _clip(grads, outs, max_norm, stream):
    same = outs is grads
    grads = list(grads)
    n = len(grads)
    if not n or not all(isinstance(g, _Tensor) for g in grads):
        raise ValueError("grads must be tensors, one at least")
    device = grads[0].device
    tensors, dtypes = grads, list(map(_dtype, grads))
    if outs is not None and not same:
        outs = list(outs)
        if len(outs) != n or not all(isinstance(o, _Tensor) for o in outs):
            raise ValueError("out must have as many tensors as grads")
        if not all(map(eq, map(_shape, outs), map(_shape, grads))):
            raise ValueError("out must have its gradients' shapes")
        tensors = grads + outs
    if device.type != "cuda" or set(map(_Tensor.get_device, tensors)) != {device.index}:
        raise ValueError("gradients and outputs must be on one GPU")
    if not all(map(_Tensor.is_contiguous, tensors)):
        raise ValueError("gradients and outputs must be contiguous")
    try:
        kinds = [_TYPES[d] for d in dtypes]
        into = kinds if tensors is grads else [_TYPES[o.dtype] for o in outs]
    except KeyError:
        raise ValueError("gradients and outputs must be float32, bfloat16 or float16") from None
    if into != kinds and any(b and a != b for a, b in zip(kinds, into)):
        raise ValueError("outputs must have their gradients' types or float32")
    other = _other(device, stream)
    if other is not None:
        with other:
            return _clip(grads, grads if same else outs, max_norm, None)
    # the fields of scd_span_t, its two types as one word
    src = list(map(_Tensor.data_ptr, grads))
    dst = src if same else [0] * n if outs is None else list(map(_Tensor.data_ptr, outs))
    words = [0] * (4 * n)
    words[0::4], words[1::4], words[2::4] = src, dst, map(_Tensor.numel, grads)
    words[3::4] = [a | b << 32 for a, b in zip(kinds, into)]
    spans = (ctypes.c_uint64 * (4 * n))(*words)
    norm = torch.empty((), dtype=torch.float32, device=device)
    need = _scratch("scd_clip_grads_workspace")
    work = torch.empty(need, dtype=torch.uint8, device=device)
    _check(lib.scd_clip_grads(spans, n, max_norm, norm.data_ptr(), work.data_ptr(), need, _current_stream(device.index)))
    return norm
