"""The operators of learned features on a machine without a GPU: the 64-bit oracle against torch's automatic
derivatives, and the refusals of the C entries, which answer before they touch a GPU."""
import ctypes
import os

import pytest
import torch

import _features_oracle as fo

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1702_07005_amd", "libscd.so")


def _gen(seed):
    return torch.Generator().manual_seed(seed)


@pytest.mark.parametrize("rows,dim", [(1, 1), (3, 7), (5, 64)])
def test_oracle_layer_norm_gradient_is_the_derivative(rows, dim):
    g = _gen(rows * 100 + dim)
    x = torch.randn(rows, dim, generator=g, dtype=torch.float64, requires_grad=True)
    w = torch.randn(dim, generator=g, dtype=torch.float64, requires_grad=True)
    b = torch.randn(dim, generator=g, dtype=torch.float64, requires_grad=True)
    dy = torch.randn(rows, dim, generator=g, dtype=torch.float64)
    y = torch.nn.functional.layer_norm(x, (dim,), w, b, 1e-5)
    y.backward(dy)
    (yo, _), (mean, _), (rstd, _) = fo.layer_norm(x.detach(), w.detach(), b.detach(), 1e-5, torch.float32)
    assert torch.allclose(yo, y.detach(), rtol=1e-12, atol=1e-12)
    (dx, _), (dw, _), (db, _) = fo.layer_norm_grad(dy, x.detach(), mean, rstd, w.detach(), torch.float32, torch.float32)
    assert torch.allclose(dx, x.grad, rtol=1e-9, atol=1e-9)
    assert torch.allclose(dw, w.grad, rtol=1e-9, atol=1e-9)
    assert torch.allclose(db, b.grad, rtol=1e-12, atol=1e-12)


def test_oracle_embed_gradient_is_the_derivative():
    g = _gen(5)
    table = torch.randn(6, 4, generator=g, dtype=torch.float64, requires_grad=True)
    tokens = torch.tensor([2, 0, 2, 5, 2])
    dy = torch.randn(5, 4, generator=g, dtype=torch.float64)
    (torch.nn.functional.embedding(tokens, table) * 3.0).backward(dy)
    v, _ = fo.embed_grad(tokens, dy, 6, 3.0, torch.float32)
    assert torch.allclose(v, table.grad, rtol=1e-14, atol=1e-14)
    v, _ = fo.embed_grad(torch.tensor([-1, 0, 6, 5, -7]), dy, 6, 1.0, torch.float32)
    assert torch.equal(v[0], dy[1]) and torch.equal(v[5], dy[3]) and not v[1:5].any()


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB):
        from paper_1702_07005_amd import build
        build.build()
    from paper_1702_07005_amd import scd
    return scd.lib


P = 0x1000  # never dereferenced: every case below fails, or has nothing to do, before any device access
F32, BF16, F16, I32, I64 = range(5)
BIG = 1 << 40


def _refused(lib, code, text, rc):
    assert rc == code and text in lib.scd_last_error().decode(), (rc, lib.scd_last_error())


def test_embed_refusals(lib):
    def call(tok=P, tt=I64, n=4, table=P, et=BF16, ts=8, rows=10, dim=8, out=P, ot=BF16, os_=8):
        return lib.scd_embed(tok, tt, n, table, et, ts, rows, dim, 1.0, out, ot, os_, None)
    for kw in (dict(tt=F32), dict(tt=7), dict(et=I32), dict(ot=-1)):
        _refused(lib, -2, "scd_embed takes", call(**kw))
    for kw in (dict(n=-1), dict(n=1 << 31), dict(rows=-1), dict(rows=1 << 31), dict(dim=0), dict(dim=(1 << 20) + 1)):
        _refused(lib, -1, "bad sizes", call(**kw))
    for kw in (dict(ts=-1), dict(os_=7)):
        _refused(lib, -1, "stride", call(**kw))
    for kw in (dict(tok=None), dict(table=None), dict(out=None)):
        _refused(lib, -1, "null device pointer", call(**kw))
    assert call(n=0, tok=None, out=None) == 0


def test_embed_grad_refusals(lib):
    def call(tok=P, tt=I64, n=4, grad=P, gt=BF16, gs=8, rows=10, dim=8, acc=0, out=P, ot=F32, os_=8, work=P, wb=BIG):
        return lib.scd_embed_grad(tok, tt, n, grad, gt, gs, rows, dim, 1.0, acc, out, ot, os_, work, wb, None)
    for kw in (dict(tt=BF16), dict(gt=I64), dict(ot=9)):
        _refused(lib, -2, "scd_embed_grad takes", call(**kw))
    for kw in (dict(n=-1), dict(n=1 << 31), dict(rows=-1), dict(rows=1 << 31), dict(dim=0), dict(dim=(1 << 20) + 1)):
        _refused(lib, -1, "bad sizes", call(**kw))
    for kw in (dict(gs=-1), dict(os_=7)):
        _refused(lib, -1, "stride", call(**kw))
    for kw in (dict(tok=None), dict(grad=None), dict(out=None)):
        _refused(lib, -1, "null device pointer", call(**kw))
    need = ctypes.c_int64()
    assert lib.scd_embed_grad_workspace(4000, 10, 8, ctypes.byref(need)) == 0 and need.value > 0
    for kw in (dict(work=None), dict(work=P + 8), dict(wb=need.value - 1)):
        _refused(lib, -1, "workspace", call(n=4000, **kw))
    assert call(rows=0, out=None) == 0
    assert call(n=0, acc=1, tok=None, grad=None, work=None) == 0
    _refused(lib, -1, "bad sizes", lib.scd_embed_grad_workspace(4, 10, 0, ctypes.byref(need)))
    assert need.value == 0
    _refused(lib, -1, "null", lib.scd_embed_grad_workspace(4, 10, 8, None))


def test_layer_norm_refusals(lib):
    def call(x=P, t=BF16, xs=8, rows=4, dim=8, w=P, b=P, pt=BF16, eps=1e-5, y=P + 64, ys=8, m=P, r=P):
        return lib.scd_layer_norm(x, t, xs, rows, dim, w, b, pt, eps, y, ys, m, r, None)
    for kw in (dict(t=I32), dict(pt=F16), dict(t=F32, pt=BF16), dict(pt=-1)):
        _refused(lib, -2, "layer norm takes", call(**kw))
    for kw in (dict(rows=-1), dict(rows=1 << 31), dict(dim=0), dict(dim=(1 << 20) + 1)):
        _refused(lib, -1, "bad sizes", call(**kw))
    for kw in (dict(eps=-1e-5), dict(eps=float("nan"))):
        _refused(lib, -1, "eps", call(**kw))
    for kw in (dict(xs=-1), dict(ys=7)):
        _refused(lib, -1, "stride", call(**kw))
    _refused(lib, -1, "in place", call(y=P, ys=9))
    for kw in (dict(x=None), dict(y=None)):
        _refused(lib, -1, "null device pointer", call(**kw))
    assert call(rows=0, x=None, y=None) == 0


def test_layer_norm_grad_refusals(lib):
    def call(dy=P, gs=8, x=P + 64, xs=8, t=BF16, m=P, r=P, rows=4, dim=8, w=P, pt=BF16, dx=P + 128, ds=8, dw=P, db=P, work=P,
             wb=BIG):
        return lib.scd_layer_norm_grad(dy, gs, x, xs, t, m, r, rows, dim, w, pt, dx, ds, dw, db, work, wb, None)
    for kw in (dict(t=I32), dict(pt=F16), dict(t=F32, pt=BF16)):
        _refused(lib, -2, "layer norm takes", call(**kw))
    for kw in (dict(rows=-1), dict(rows=1 << 31), dict(dim=0), dict(dim=(1 << 20) + 1)):
        _refused(lib, -1, "bad sizes", call(**kw))
    for kw in (dict(xs=-1), dict(gs=-1), dict(ds=7)):
        _refused(lib, -1, "stride", call(**kw))
    for kw in (dict(dx=P, ds=9), dict(dx=P + 64, ds=9)):
        _refused(lib, -1, "in place", call(**kw))
    for kw in (dict(dw=None), dict(db=None)):
        _refused(lib, -1, "go together", call(**kw))
    for kw in (dict(dy=None), dict(x=None), dict(m=None), dict(r=None), dict(dx=None)):
        _refused(lib, -1, "null device pointer", call(**kw))
    need = ctypes.c_int64()
    assert lib.scd_layer_norm_grad_workspace(4, 8, ctypes.byref(need)) == 0 and need.value > 0
    for kw in (dict(work=None), dict(work=P + 8), dict(wb=need.value - 1)):
        _refused(lib, -1, "workspace", call(**kw))
    _refused(lib, -1, "null", lib.scd_layer_norm_grad_workspace(4, 8, None))


class _Span(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("n", ctypes.c_int64), ("src_type", ctypes.c_int32),
                ("dst_type", ctypes.c_int32)]


def test_clip_refusals(lib):
    def call(span=(P, P, 4, BF16, BF16), count=1, most=1.0, norm=P, work=P, wb=BIG):
        s = _Span(*span)
        return lib.scd_clip_grads(ctypes.byref(s) if count else None, count, most, norm, work, wb, None)
    _refused(lib, -1, "bad spans", call(count=-1))
    _refused(lib, -1, "bad spans", lib.scd_clip_grads(None, 1, 1.0, P, P, BIG, None))
    for most in (-1.0, float("nan")):
        _refused(lib, -1, "max_norm", call(most=most))
    _refused(lib, -1, "null device pointer", call(norm=None))
    for span in ((P, P, 4, I32, I32), (P, P + 64, 4, F32, BF16), (P, P + 64, 4, F16, BF16)):
        _refused(lib, -2, "span 0", call(span=span))
    for span in ((P, P, -1, F32, F32), (None, P, 1, F32, F32), (P, P, 1 << 62, F32, F32)):
        _refused(lib, -1, "span 0", call(span=span))
    _refused(lib, -1, "in place", call(span=(P, P, 4, BF16, F32)))
    need = ctypes.c_int64()
    assert lib.scd_clip_grads_workspace(ctypes.byref(need)) == 0 and need.value > 0
    for kw in (dict(work=None), dict(work=P + 8), dict(wb=need.value - 1)):
        _refused(lib, -1, "workspace", call(**kw))
    _refused(lib, -1, "null", lib.scd_clip_grads_workspace(None))
