"""Operators of learned features: table lookup, layer norm, their gradients, and gradient clipping.

They serve models whose coordinates are rows of a learned table instead of one-hot columns: ids are
looked up, the vectors normalised, a linear read-out is fitted on them by ``scd.Solver``, and the table is
trained by the read-out's gradient.  Every step runs in the HIP kernels of ``libscd.so`` (``include/scd.h``
documents the calls).  The compiled binding ``_features.so`` checks arguments and allocates outputs and scratch
from torch's caching allocator, so the calls enqueue on a stream, never synchronise, and can be captured in
graphs.  There is no fallback: if the binding is not built this module raises on import.

Matrices may be views with any row stride, but their last dimension has unit stride.  Work is enqueued on
the current stream, or on ``stream`` (a torch stream or a raw handle), with which the caller orders the
inputs; outputs that the call allocates then belong to that stream, and the other tensors may be dropped once the call
returns.

The operators are outside autograd: they record nothing, results never require gradients, and backward passes are
calls of their own.  Tensors that a call writes to (``out``, gradients clipped in place) count it as an in-place
operation, so that autograd refuses a backward pass that needs their former values; one that itself requires gradients is
refused unless gradients are off (``torch.no_grad()``).

    x = features.embed(ids, table, scale=table.shape[1] ** 0.5)
    y, mean, rstd = features.layer_norm(x, weight, bias)
    dx, dw, db = features.layer_norm_grad(dy, x, mean, rstd, weight)
    dtable = features.embed_grad(ids, dx, table.shape[0], scale=table.shape[1] ** 0.5)
    norm = features.clip_grads([dtable, dw, db], 1.0)
"""
from __future__ import annotations

import os

import torch

from . import scd  # noqa: F401  (loads libscd.so)

if not os.path.exists(os.path.join(os.path.dirname(os.path.abspath(__file__)), "_features.so")):
    raise ImportError("_features.so is not built: run `python -m paper_1702_07005_amd.build`")
from . import _features  # noqa: E402

_device = torch._C._cuda_getDevice
_stream = torch._C._cuda_getCurrentRawStream


def _elsewhere(tensor, stream, call, *args):
    """Makes the call on the tensor's device, or on a given stream, by making that the current one.  The memory of tensors
    that belong to another stream is not given away before the given one is done with them."""
    if not (isinstance(tensor, torch.Tensor) and tensor.is_cuda):
        raise ValueError("CUDA tensors are needed")
    if stream is None:
        context = torch.cuda.device(tensor.device)
    else:
        if not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(int(stream), device=tensor.device)
        if stream.device != tensor.device:
            raise ValueError(f"the stream is on {stream.device}, the tensors on {tensor.device}")
        context = torch.cuda.stream(stream)
        for a in args:
            for t in a if isinstance(a, (list, tuple)) else (a,):
                if isinstance(t, torch.Tensor) and t.is_cuda:
                    t.record_stream(stream)
    with context:
        return call(*args)


def embed(tokens, table, scale=1.0, out=None, dtype=None, stream=None):
    """``out[..., :] = scale * table[tokens[...], :]``; a negative token (a padded place) gives zeros, one of
    at least ``table.shape[0]`` NaN.

    ``tokens``: contiguous int32 or int64, any shape; ``table``: [rows, dim] of float32, bfloat16 or float16;
    ``dtype``: of the output (the table's by default)."""
    if stream is None:
        d = _device()
        result = _features.embed(d, _stream(d), tokens, table, scale, out, dtype)
        if result is not None:
            return result
    return _elsewhere(table, stream, embed, tokens, table, scale, out, dtype)


def embed_grad(tokens, grad, rows, scale=1.0, out=None, accumulate=False, dtype=None, stream=None):
    """The gradient of ``embed`` with respect to its table: row v of [rows, dim] is ``scale`` times the sum of
    ``grad``'s rows whose token is v.  Tokens outside [0, rows) add to nothing.  ``accumulate`` adds to
    ``out`` instead of overwriting it.

    ``grad``: [*tokens.shape, dim]; ``dtype``: of the result (``grad``'s by default).  The result is
    bit-identical from call to call."""
    if stream is None:
        d = _device()
        result = _features.embed_grad(d, _stream(d), tokens, grad, rows, scale, out, accumulate, dtype)
        if result is not None:
            return result
    return _elsewhere(grad, stream, embed_grad, tokens, grad, rows, scale, out, accumulate, dtype)


def layer_norm(x, weight=None, bias=None, eps=1e-5, out=None, stream=None):
    """``(x - mean) * rstd * weight + bias`` over the last dimension; returns it with ``mean`` and ``rstd``
    (float32, one for each row), which ``layer_norm_grad`` takes.

    ``weight`` and ``bias``: [dim], both of ``x``'s type or both float32, or None.  ``out`` may be ``x``."""
    if stream is None:
        d = _device()
        result = _features.layer_norm(d, _stream(d), x, weight, bias, eps, out)
        if result is not None:
            return result
    return _elsewhere(x, stream, layer_norm, x, weight, bias, eps, out)


def layer_norm_grad(grad, x, mean, rstd, weight=None, params=True, out=None, stream=None):
    """The gradients of ``layer_norm`` with respect to ``x``, ``weight`` and ``bias``, from the gradient of its
    output and the ``mean`` and ``rstd`` it returned.  Those of weight and bias have the weight's type (``x``'s
    where there is none) and are None with ``params=False``.  ``out`` (for ``x``'s) may be ``grad`` or ``x``."""
    if stream is None:
        d = _device()
        result = _features.layer_norm_grad(d, _stream(d), grad, x, mean, rstd, weight, params, out)
        if result is not None:
            return result
    return _elsewhere(x, stream, layer_norm_grad, grad, x, mean, rstd, weight, params, out)


def clip_grads(grads, max_norm, out=None, stream=None):
    """Scales the tensors of ``grads`` together so that their norm is at most ``max_norm``, in place or into the
    tensors of ``out`` (each of its gradient's type or float32).  Returns the norm before, a float32 tensor on
    the GPU, without waiting for it.

    The tensors are contiguous, of float32, bfloat16 or float16, and on one device.  Those that are written to share no
    memory with others of the call."""
    grads = grads if isinstance(grads, (list, tuple)) else list(grads)
    return _clip(grads, grads if out is None else out, max_norm, stream)


def grad_norm(grads, stream=None):
    """The norm of all tensors of ``grads`` together: a float32 tensor on the GPU."""
    grads = grads if isinstance(grads, (list, tuple)) else list(grads)
    return _clip(grads, None, float("inf"), stream)


def _clip(grads, outs, max_norm, stream):
    if stream is None:
        d = _device()
        result = _features.clip(d, _stream(d), grads, outs, max_norm)
        if result is not None:
            return result
    return _elsewhere(grads[0] if grads else None, stream, _clip, grads, outs, max_norm, None)
