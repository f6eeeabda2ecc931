"""Operators of learned features: table lookup, layer and root-mean-square norm, their gradients, gradient clipping, and
the AdamW step.

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

With the root-mean-square norm, and with a step of AdamW that clips on the way:

    y, rstd, h = features.rms_norm(x, weight, residual)
    dh, dw = features.rms_norm_grad(dy, h, rstd, weight)
    params, grads = [table, weight], [dtable, dw]
    state = features.adamw_state(params, bits=8)  # once
    features.adamw(params, grads, state, step, lr=1e-3, norm=features.grad_norm(grads), max_norm=1.0)
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
        _record(args, stream)
    with context:
        return call(*args)


def _record(a, stream):
    if isinstance(a, torch.Tensor):
        if a.is_cuda:
            a.record_stream(stream)
    elif isinstance(a, (list, tuple)):
        for t in a:
            _record(t, stream)


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


def rms_norm(x, weight=None, residual=None, eps=1e-6, out=None, sum_out=None, stream=None):
    """``h * rstd * weight`` over the last dimension, with ``h = x + residual`` and ``rstd = 1 / sqrt(mean(h ** 2) + eps)``;
    returns it with ``rstd`` (float32, one for each row) and ``h``, which ``rms_norm_grad`` takes.

    The sum is rounded to ``x``'s type and normalised as it is kept; without a residual ``h`` is ``x`` (detached if it requires
    gradients), or None where ``out`` takes ``x``'s place.  ``residual``: of ``x``'s type and shape; ``weight``: [dim], of
    ``x``'s type or float32, or None.  ``out`` and ``sum_out`` (for ``h``) may be ``x`` or ``residual``, but not the same."""
    if stream is None:
        d = _device()
        result = _features.rms_norm(d, _stream(d), x, weight, residual, eps, out, sum_out, None)
        if result is not None:
            return result
    return _elsewhere(x, stream, rms_norm, x, weight, residual, eps, out, sum_out)


def rms_norm_8bit(x, weight=None, residual=None, eps=1e-6, group=None, out=None, sum_out=None, stream=None):
    """``rms_norm`` with its result in 8 bits (``torch.float8_e4m3fn``) and scales; returns both with ``rstd`` and ``h``.

    What the 8 bits stand for is their value times the scale: the largest magnitude of the row, or of each ``group`` (32, 64
    or 128) columns, over 448.  ``scale``: float32, of ``x``'s leading shape, with a group [..., ceil(dim / group)].  The
    result is rounded once, from 32 bits.  ``out``: of 8 bits, any row stride."""
    if stream is None:
        d = _device()
        result = _features.rms_norm(d, _stream(d), x, weight, residual, eps, out, sum_out, _columns(group))
        if result is not None:
            return result
    return _elsewhere(x, stream, rms_norm_8bit, x, weight, residual, eps, group, out, sum_out)


def _columns(group):
    if group is None:
        return 0
    if group not in (32, 64, 128):
        raise ValueError("group must be None, 32, 64 or 128")
    return int(group)


def rms_norm_grad(grad, x, rstd, weight=None, residual_grad=None, params=True, out=None, stream=None):
    """The gradients of ``rms_norm`` with respect to ``h`` (which is that of ``x`` and of ``residual`` alike) and ``weight``,
    from the gradient of its output and the ``h`` (here ``x``) and ``rstd`` it returned.

    ``residual_grad``, the gradient that reaches ``h`` another way, is added before the result is rounded.  The weight's has
    its type (``x``'s where there is none) and is None with ``params=False``.  ``out`` may be any of the three matrices."""
    if stream is None:
        d = _device()
        result = _features.rms_norm_grad(d, _stream(d), grad, x, rstd, weight, residual_grad, params, out)
        if result is not None:
            return result
    return _elsewhere(x, stream, rms_norm_grad, grad, x, rstd, weight, residual_grad, params, out)


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


STATE_BLOCK = 256  # consecutive elements of a parameter whose states of 8 bits share a scale


def adamw_state(params, bits=32):
    """The states of ``params`` before the first step of ``adamw``, a tuple for each: the averages of the gradient and of its
    square (float32), or with ``bits=8`` the average and the square root of the other (``torch.float8_e4m3fn``), then the
    scales of both (float32, one for each 256 consecutive elements): what they stand for is their value times the scale."""
    if bits not in (32, 8):
        raise ValueError("bits must be 32 or 8")

    def zeros(p):
        if bits == 32:
            return tuple(torch.zeros(p.shape, dtype=torch.float32, device=p.device) for _ in range(2))
        blocks = (p.numel() + STATE_BLOCK - 1) // STATE_BLOCK
        codes = [torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn) for _ in range(2)]
        return (*codes, *(torch.zeros(blocks, dtype=torch.float32, device=p.device) for _ in range(2)))

    return [zeros(p) for p in params]


def adamw(params, grads, state, step, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, norm=None, max_norm=1.0, copies=None,
          seed=0, stream=None):
    """One AdamW step of all ``params`` together, in place, by ``grads`` and ``state`` (from ``adamw_state``; updated):

        g = grad * min(1, max_norm / norm);  m = b1 * m + (1 - b1) * g;  v = b2 * v + (1 - b2) * g ** 2
        param = param * (1 - lr * weight_decay) - lr * (m / (1 - b1 ** step)) / (sqrt(v / (1 - b2 ** step)) + eps)

    ``params``: float32 with gradients of any type, or bfloat16 or float16 with gradients of that type or float32; tensors are
    contiguous and on one device, and those that are written to share no memory with others of the call.  Parameters that
    require gradients are updated under ``torch.no_grad()``.  ``step`` counts from 1.  It and ``lr`` may be tensors of one
    element on the GPU (int64, float32), which a captured call reads at every replay.  ``weight_decay``: a number, or one for
    each parameter.  ``norm``: that of all gradients, as ``grad_norm`` returns it, or None for no clipping.  ``copies``:
    bfloat16 or float16 tensors (None for none) that receive the new float32 parameters.

    States of 8 bits are rounded up or down at random, by a hash of ``seed``, ``step`` and the element's place, so that
    small changes add up.  They cost 4 bytes of traffic an element instead of 16."""
    if not (isinstance(params, list) and isinstance(grads, list) and isinstance(state, list) and isinstance(weight_decay, float)):
        params, grads, state = list(params), list(grads), list(state)
        if not isinstance(weight_decay, (int, float)):
            weight_decay = list(weight_decay)
    if copies is not None:
        copies = list(copies)
    _adamw(params, grads, state, step, lr, *betas, eps, weight_decay, norm, max_norm, copies, seed, stream)


def _adamw(*args):
    *args, stream = args
    if stream is None:
        d = _device()
        if _features.adamw(d, _stream(d), *args) is not None:
            return True
    return _elsewhere(args[0][0] if args[0] else None, stream, _adamw, *args, None)
