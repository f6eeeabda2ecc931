"""The root-mean-square norm and the AdamW step on a machine without a GPU: their 64-bit oracle against torch's automatic
derivatives and its optimizer, the rounding to 8 bits against its means, and the refusals of the C entries, which answer
before they touch a GPU."""
import ctypes
import os

import pytest
import torch

import _training_oracle as to

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1702_07005_amd", "libscd.so")


def _gen(seed):
    return torch.Generator().manual_seed(seed)


@pytest.mark.parametrize("rows,dim", [(1, 1), (3, 7), (5, 64)])
def test_oracle_rms_gradient_is_the_derivative(rows, dim):
    g = _gen(rows * 100 + dim)
    x, res, dy, more = (torch.randn(rows, dim, generator=g, dtype=torch.float64) for _ in range(4))
    w = torch.randn(dim, generator=g, dtype=torch.float64, requires_grad=True)
    x.requires_grad_()
    res.requires_grad_()
    h = x + res
    y = h * (h.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * w
    ((y * dy).sum() + (h * more).sum()).backward()
    (yo, _), (rstd, _) = to.rms_norm(h.detach(), w.detach(), 1e-6)
    assert torch.allclose(yo, y.detach(), rtol=1e-12, atol=1e-12)
    (dx, _), (dw, _) = to.rms_norm_grad(dy, h.detach(), rstd, w.detach(), more, torch.float64, torch.float64)
    assert torch.allclose(dx, x.grad, rtol=1e-9, atol=1e-9) and torch.equal(x.grad, res.grad)
    assert torch.allclose(dw, w.grad, rtol=1e-9, atol=1e-9)


def test_oracle_adamw_is_torchs():
    g = _gen(3)
    p = torch.randn(37, generator=g, dtype=torch.float64, requires_grad=True)
    opt = torch.optim.AdamW([p], lr=1e-2, betas=(0.8, 0.99), eps=1e-6, weight_decay=0.1)
    mine, state = p.detach().clone(), (torch.zeros(37), torch.zeros(37))
    for t in range(1, 6):
        grad = torch.randn(37, generator=g, dtype=torch.float64)
        norm = float(grad.norm())
        p.grad = grad / norm
        opt.step()
        out = to.adamw(mine, grad, state, t, 1e-2, (0.8, 0.99), 1e-6, 0.1, norm=norm, max_norm=1.0)
        mine, state = out["param"][0], (out["m"][0], out["v"][0])
        assert torch.allclose(mine, p.detach(), rtol=1e-12, atol=1e-14)


def test_values_of_8_bits_are_the_grid():
    every = torch.arange(256, dtype=torch.uint8).view(to.E4M3).float()
    every = every[torch.isfinite(every) & (every >= 0)].double().unique()
    assert every.numel() == 127 and float(every[-1]) == to.TOP
    # neighbours lie as far apart as the grid says, above a value and up to the next
    assert torch.equal(every[1:] - every[:-1], to.grid(every[:-1])) and torch.equal(to.grid((every[1:] + every[:-1]) / 2), to.grid(every[:-1]))


def test_random_rounding_keeps_the_means():
    z = torch.tensor([0.0, 2.0 ** -9, 3.3e-3, 0.01, 0.07, 1.0, 1.03, 17.7, 300.0, 447.0, 448.0], dtype=torch.float64)
    u = (torch.arange(65536, dtype=torch.float64)[:, None] + 0.5) / 65536
    m, r = to.round_m(z.expand(65536, -1), u.expand(-1, z.numel())), to.round_r(z.expand(65536, -1), u.expand(-1, z.numel()))
    # u is spread evenly, so that the means are off by at most 2^-16 of a step
    assert ((m.mean(0) - z).abs() <= 2.0 ** -16 * to.grid(z)).all()
    far = z >= 2.0 ** -9
    assert ((r.square().mean(0) - z.square()).abs() <= 2.0 ** -16 * 2 * to.grid(z) * (z + to.grid(z)))[far].all()
    assert (r[:, ~far & (z > 0)] == 2.0 ** -9).all() and (r[:, z == 0] == 0).all()
    assert torch.equal(m.float().to(to.E4M3).double(), m) and torch.equal(r.float().to(to.E4M3).double(), r)


def test_words_are_spread_evenly_and_differ():
    w = to.words(1 << 16, 7, 3, 0)
    for part in (w & 0xFF, (w >> 8) & 0xFF, (w >> 16) & 0xFF, w >> 24):
        counts = torch.bincount(part, minlength=256).double()
        # 256 of each expected, standard deviation 16: 6 of them
        assert ((counts - 256).abs() <= 96).all()
    for other in (to.words(1 << 16, 8, 3, 0), to.words(1 << 16, 7, 4, 0), to.words(1 << 16, 7, 3, 1)):
        assert (w == other).double().mean() < 1e-3
    assert not torch.equal(to.words(9, 7, 3, 0, start=1 << 32), w[:9])


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB):
        from paper_1702_07005_amd import build
        build.build()
    from paper_1702_07005_amd import scd
    return scd.lib


P = 0x1000  # never dereferenced: every case below fails, or has nothing to do, before any device access
F32, BF16, F16, I32, I64, E4M3 = range(6)
BIG = 1 << 40
INF, NAN = float("inf"), float("nan")


def _refused(lib, code, text, rc):
    assert rc == code and text in lib.scd_last_error().decode(), (rc, lib.scd_last_error())


def test_rms_norm_refusals(lib):
    def call(x=P, t=BF16, xs=8, res=P + 64, rs=8, rows=4, dim=8, w=P, pt=BF16, eps=1e-6, y=P + 128, yt=BF16, ys=8, scale=P, group=0, sum_=P + 256, ss=8, r=P):
        return lib.scd_rms_norm(x, t, xs, res, rs, rows, dim, w, pt, eps, y, yt, ys, scale, group, sum_, ss, r, None)
    for kw in (dict(t=I32), dict(t=E4M3), dict(pt=F16), dict(t=F32, pt=BF16, yt=F32), dict(pt=-1)):
        _refused(lib, -2, "rms norm takes", call(**kw))
    for kw in (dict(yt=F32), dict(yt=F16), dict(yt=9)):
        _refused(lib, -2, "rms norm gives", call(**kw))
    for kw in (dict(rows=-1), dict(rows=1 << 31), dict(dim=0), dict(dim=(1 << 20) + 1)):
        _refused(lib, -1, "bad sizes", call(**kw))
    for kw in (dict(eps=-1e-5), dict(eps=NAN)):
        _refused(lib, -1, "eps", call(**kw))
    for kw in (dict(group=32), dict(yt=E4M3, group=16), dict(yt=E4M3, group=-128), dict(yt=E4M3, group=256), dict(yt=E4M3, group=1 << 32)):
        _refused(lib, -1, "group", call(**kw))
    for kw in (dict(xs=-1), dict(rs=-1), dict(ys=7), dict(ss=7)):
        _refused(lib, -1, "stride", call(**kw))
    for kw in (dict(y=P, ys=9), dict(y=P + 64, ys=9), dict(sum_=P, ss=9), dict(sum_=P + 64, ss=9), dict(x=P, xs=0, y=P)):
        _refused(lib, -1, "in place", call(**kw))
    for kw in (dict(sum_=P + 128), dict(yt=E4M3, y=P), dict(yt=E4M3, y=P + 64)):
        _refused(lib, -1, "overlap", call(**kw))
    for kw in (dict(x=None), dict(y=None), dict(sum_=None), dict(yt=E4M3, scale=None)):
        _refused(lib, -1, "null device pointer", call(**kw))
    assert call(rows=0, x=None, res=None, y=None, sum_=None, r=None) == 0
    assert call(rows=0, yt=E4M3, group=64, x=None, y=None, scale=None) == 0


def test_rms_norm_grad_refusals(lib):
    def call(dy=P, gs=8, h=P + 64, hs=8, t=BF16, r=P, rows=4, dim=8, w=P, pt=BF16, res=P + 128, rs=8, dh=P + 256, ds=8, dw=P, work=P, wb=BIG):
        return lib.scd_rms_norm_grad(dy, gs, h, hs, t, r, rows, dim, w, pt, res, rs, dh, ds, dw, work, wb, None)
    for kw in (dict(t=I32), dict(pt=F16), dict(t=F32, pt=BF16)):
        _refused(lib, -2, "rms norm takes", call(**kw))
    for kw in (dict(rows=-1), dict(rows=1 << 31), dict(dim=0), dict(dim=(1 << 20) + 1)):
        _refused(lib, -1, "bad sizes", call(**kw))
    for kw in (dict(gs=-1), dict(hs=-1), dict(rs=-1), dict(ds=7)):
        _refused(lib, -1, "stride", call(**kw))
    for kw in (dict(dh=P, ds=9), dict(dh=P + 64, ds=9), dict(dh=P + 128, ds=9)):
        _refused(lib, -1, "in place", call(**kw))
    for kw in (dict(dy=None), dict(h=None), dict(r=None), dict(dh=None)):
        _refused(lib, -1, "null device pointer", call(**kw))
    need = ctypes.c_int64()
    assert lib.scd_rms_norm_grad_workspace(4, 8, ctypes.byref(need)) == 0 and need.value > 0
    for kw in (dict(work=None), dict(work=P + 8), dict(wb=need.value - 1)):
        _refused(lib, -1, "workspace", call(**kw))
    assert lib.scd_rms_norm_grad_workspace(1, 8, ctypes.byref(need)) == 0 and need.value == 0
    _refused(lib, -1, "null", lib.scd_rms_norm_grad_workspace(4, 8, None))
    _refused(lib, -1, "bad sizes", lib.scd_rms_norm_grad_workspace(4, 0, ctypes.byref(need)))
    assert call(rows=0, dy=None, h=None, r=None, dh=None, dw=None, work=None, wb=0) == 0


class _Span(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p), ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("copy", ctypes.c_void_p), ("n", ctypes.c_int64), ("weight_decay", ctypes.c_float),
                ("param_type", ctypes.c_int32), ("grad_type", ctypes.c_int32), ("state_type", ctypes.c_int32), ("copy_type", ctypes.c_int32)]


class _Options(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double), ("step", ctypes.c_int64),
                ("lr_dev", ctypes.c_void_p), ("step_dev", ctypes.c_void_p), ("norm_dev", ctypes.c_void_p), ("max_norm", ctypes.c_float), ("seed", ctypes.c_uint32)]


def test_adamw_refusals(lib):
    def call(n=4, param=P, grad=P, m=P, v=P, ms=P, vs=P, copy=None, decay=0.0, pt=F32, gt=F32, st=F32, ct=BF16, count=1, **options):
        span = _Span(param, grad, m, v, ms, vs, copy, n, decay, pt, gt, st, ct)
        o = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, lr_dev=None, step_dev=None, norm_dev=None, max_norm=1.0, seed=0)
        o.update(options)
        return lib.scd_adamw(ctypes.byref(span) if count else None, count, ctypes.byref(_Options(**o)), None)
    _refused(lib, -1, "bad spans", call(count=-1))
    _refused(lib, -1, "bad spans", lib.scd_adamw(None, 1, ctypes.byref(_Options()), None))
    _refused(lib, -1, "options", lib.scd_adamw(ctypes.byref(_Span()), 1, None, None))
    for lr in (-1e-3, NAN, INF):
        _refused(lib, -1, "lr", call(lr=lr))
    for kw in (dict(beta1=1.0), dict(beta2=1.0), dict(beta1=-0.1), dict(beta2=NAN)):
        _refused(lib, -1, "betas", call(**kw))
    for eps in (-1e-8, NAN, INF):
        _refused(lib, -1, "eps", call(eps=eps))
    for step in (0, -3):
        _refused(lib, -1, "step", call(step=step))
    for most in (-1.0, NAN):
        _refused(lib, -1, "max_norm", call(norm_dev=P, max_norm=most))
    for kw in (dict(pt=I32), dict(gt=E4M3), dict(pt=BF16, gt=F16), dict(pt=F16, gt=BF16)):
        _refused(lib, -2, "float32 parameters", call(**kw))
    for st in (BF16, F16, I32):
        _refused(lib, -2, "states", call(st=st))
    for kw in (dict(copy=P, ct=F32), dict(copy=P, pt=BF16, gt=BF16)):
        _refused(lib, -2, "copies", call(**kw))
    for decay in (-0.1, NAN, INF):
        _refused(lib, -1, "weight_decay", call(decay=decay))
    for kw in (dict(n=-1), dict(n=1 << 62), dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(st=E4M3, ms=None), dict(st=E4M3, vs=None)):
        _refused(lib, -1, "span 0", call(**kw))
    # nothing to do, and what is not used is not looked at
    assert call(count=0) == 0
    assert call(n=0, param=None, grad=None, m=None, v=None) == 0
    assert call(n=0, lr=NAN, lr_dev=P, step=0, step_dev=P, max_norm=NAN) == 0
