"""The root-mean-square norm, its output in 8 bits and its gradient on the GPU against their 64-bit oracle
(tests/_training_oracle.py), at the sizes, strides, types and places where they can go wrong."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import _features_oracle as fo  # noqa: E402
import _training_oracle as to  # noqa: E402
from paper_1702_07005_amd import features, scd  # noqa: E402

DEV = "cuda"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
PAIRS = [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)]
EPS = float(torch.tensor(1e-6))
# Both sides of every group of lanes: one vector a lane from 4 to 64, two to four in a wave, two or four waves and more, and
# rows that are read again.
DIMS = [1, 3, 4, 7, 8, 9, 16, 31, 32, 33, 63, 65, 127, 129, 255, 257, 511, 513, 777, 1025, 1536, 1540, 2049, 2500, 3077, 4097, 5000, 6000, 6150, 8193, 10_001, 12_000, 12_300,
        16_384, 16_385, 40_001]


@pytest.fixture(scope="module", autouse=True)
def _give_back_memory():
    yield
    torch.cuda.empty_cache()


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _normal(g, *shape, dtype=F32, std=1.0):
    return (torch.randn(*shape, generator=g) * std).to(dtype)


def _rows_of_sizes(g, rows, dim, dtype):
    return (_normal(g, rows, dim) * (0.1 + 2 * torch.rand(rows, 1, generator=g)) + 0.1).to(dtype)


def _strided(t, pad, offset=0):
    """A device copy whose rows lie `pad` elements further apart and begin `offset` elements into the memory."""
    n, d = t.shape
    room = torch.full((offset + n * (d + pad) + 8,), float("nan"), device=DEV).to(t.dtype)
    v = room[offset:offset + n * (d + pad)].view(n, d + pad)[:, :d]
    v.copy_(t)
    return v


def _untouched(v):
    """The elements between the rows of a view made by `_strided` are still NaN."""
    n, d = v.shape
    whole = v.as_strided((n, v.stride(0)), (v.stride(0), 1), v.storage_offset())
    return bool(torch.isnan(whole[:, d:].float()).all())


def _close8(got, want, what):
    """Values of 8 bits within half a step of the value, and the bound of what they are rounded from."""
    value, bound = want
    got = got.cpu().float().double()
    assert not torch.isnan(got).any()
    bad = (got - value).abs() > bound
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside; {got[bad][0]} for {value[bad][0]} within {bound[bad][0]}"


def _check(rows, dim, x_type, p_type, residual, seed=0, groups=(None, 32, 64, 128), with_weight=True):
    g = _gen(seed + rows * 31 + dim)
    x = _rows_of_sizes(g, rows, dim, x_type)
    res = _rows_of_sizes(g, rows, dim, x_type) if residual else None
    w = (1 + _normal(g, dim, std=0.3)).to(p_type) if with_weight else None
    xd, wd, rd = x.to(DEV), None if w is None else w.to(DEV), None if res is None else res.to(DEV)
    y, rstd, h = features.rms_norm(xd, wd, rd)
    want_h = to.stream(x, res)
    want_y, want_rstd = to.rms_norm(want_h, w, EPS)
    if residual:
        assert torch.equal(h.cpu(), want_h) and torch.equal(xd.cpu(), x) and torch.equal(rd.cpu(), res)
    else:
        assert h is xd
    fo.close(y, want_y, "y")
    fo.close(rstd, want_rstd, "rstd")
    for group in groups:
        q, scale, rstd8, h8 = features.rms_norm_8bit(xd, wd, rd, group=group)
        assert q.dtype == torch.float8_e4m3fn and torch.equal(rstd8, rstd) and torch.equal(h8, h)
        want_q, want_scale = to.rms_norm_8bit(want_h, w, EPS, group)
        assert scale.shape == ((rows,) if group is None else (rows, -(-dim // group)))
        fo.close(scale, want_scale, f"scale {group}")
        _close8(q, want_q, f"q {group}")
    return xd, wd, h, rstd


def _check_grad(rows, dim, x_type, p_type, residual, seed=0, with_weight=True):
    g = _gen(seed + rows * 37 + dim)
    h, dy = _rows_of_sizes(g, rows, dim, x_type), _normal(g, rows, dim, dtype=x_type)
    more = _normal(g, rows, dim, dtype=x_type) if residual else None
    w = (1 + _normal(g, dim, std=0.3)).to(p_type) if with_weight else None
    _, rstd, _ = features.rms_norm(h.to(DEV), None if w is None else w.to(DEV))
    args = (dy.to(DEV), h.to(DEV), rstd, None if w is None else w.to(DEV), None if more is None else more.to(DEV))
    dh, dw = features.rms_norm_grad(*args)
    want_dh, want_dw = to.rms_norm_grad(dy, h, rstd.cpu(), w, more, x_type, p_type if with_weight else x_type)
    fo.close(dh, want_dh, "dh")
    fo.close(dw, want_dw, "dw")
    again = features.rms_norm_grad(*args)
    assert torch.equal(again[0], dh) and torch.equal(again[1], dw)
    alone, none = features.rms_norm_grad(*args, params=False)
    assert none is None and torch.equal(alone, dh)


@pytest.mark.parametrize("x,p", PAIRS)
@pytest.mark.parametrize("dim", DIMS)
def test_rms_norm_widths(dim, x, p):
    rows = 5 if dim > 2000 else 37
    _check(rows, dim, x, p, residual=True)
    _check(rows, dim, x, p, residual=False, groups=(None, 128))


@pytest.mark.parametrize("x,p", PAIRS)
@pytest.mark.parametrize("dim", DIMS)
def test_rms_norm_gradient_widths(dim, x, p):
    rows = 5 if dim > 2000 else 37
    _check_grad(rows, dim, x, p, residual=True)
    _check_grad(rows, dim, x, p, residual=False)


# One row, several for each group of lanes and several turns of the rows' loop, one more or one less than they divide.
@pytest.mark.parametrize("rows,dim", [(1, 64), (1, 4096), (2, 4096), (255, 16), (2049, 24), (5003, 40), (3001, 300), (700, 1500), (9001, 5), (131_073, 9),
                                      (4097, 1030), (2051, 5000)])
def test_rms_norm_rows(rows, dim):
    _check(rows, dim, BF16 if dim % 2 else F32, F32, residual=bool(rows % 2), groups=(None, 32))
    _check_grad(rows, dim, BF16 if dim % 2 else F32, F32, residual=bool(rows % 2))


# One workgroup does few rows for each of its groups alone; one row needs no workspace in any case.
@pytest.mark.parametrize("x", [F32, BF16])
@pytest.mark.parametrize("rows,dim", [(1, 5), (64, 30), (65, 30), (8, 700), (9, 700), (16, 700), (17, 700), (2, 5000), (3, 5000), (1, 33_000), (2, 33_000),
                                      (3, 33_000), (70, 33_000)])
def test_rms_norm_gradient_of_few_rows(x, rows, dim):
    _check_grad(rows, dim, x, F32, residual=True)


@pytest.mark.parametrize("dim", [20, 513, 17_000])
def test_rms_norm_without_weight_in_views_and_in_place(dim):
    _check(11, dim, BF16, BF16, residual=True, with_weight=False)
    _check_grad(11, dim, BF16, BF16, residual=True, with_weight=False)
    g = _gen(dim)
    rows = 11
    x, res, dy, more = (_rows_of_sizes(g, rows, dim, BF16) for _ in range(4))
    w = (1 + _normal(g, dim, std=0.3)).to(BF16).to(DEV)
    y, rstd, h = features.rms_norm(x.to(DEV), w, res.to(DEV))
    q, scale, _, _ = features.rms_norm_8bit(x.to(DEV), w, res.to(DEV), group=64)
    q0, scale0, _, _ = features.rms_norm_8bit(x.to(DEV), w, res.to(DEV))
    xv, rv, yv, sv = _strided(x, 7, 1), _strided(res, 2, 3), _strided(x, 3, 5), _strided(x, 9)
    got = features.rms_norm(xv, w, rv, out=yv, sum_out=sv)
    assert got[0] is yv and got[2] is sv and _untouched(yv) and _untouched(sv)
    assert torch.equal(yv, y) and torch.equal(sv, h) and torch.equal(got[1], rstd)
    qv = torch.full((rows, dim + 5), float("nan"), device=DEV).to(torch.float8_e4m3fn)[:, 2:dim + 2]
    for group, want, want_scale in ((64, q, scale), (None, q0, scale0)):
        got = features.rms_norm_8bit(xv, w, rv, group=group, out=qv)
        assert got[0] is qv and torch.equal(qv.float(), want.float()) and torch.equal(got[1], want_scale)
        whole = qv.as_strided((rows, dim + 5), (dim + 5, 1), 0).float()
        assert torch.isnan(whole[:, :2]).all() and torch.isnan(whole[:, dim + 2:]).all()
    # the stream is updated in its place, the result takes x's, or the other way round
    for out, total in ((0, 1), (1, 0)):
        place = [_strided(x, 7, 1), _strided(res, 2, 3)]
        got = features.rms_norm(place[0], w, place[1], out=place[out], sum_out=place[total])
        assert _untouched(place[0]) and _untouched(place[1]) and torch.equal(place[out], y) and torch.equal(place[total], h) and torch.equal(got[1], rstd)
    place = _strided(res, 2, 3)
    got = features.rms_norm_8bit(x.to(DEV), w, place, sum_out=place)
    assert torch.equal(got[0].float(), q0.float()) and torch.equal(place, h)
    # without a residual, in place
    plain = features.rms_norm(x.to(DEV), w)
    got = features.rms_norm(xv, w, out=xv)
    assert got[0] is xv and _untouched(xv) and torch.equal(xv, plain[0]) and torch.equal(got[1], plain[1])
    # leading dimensions, one vector, one residual for all rows
    three = features.rms_norm(x.to(DEV).view(rows, 1, dim), w, res.to(DEV).view(rows, 1, dim))
    assert three[0].shape == (rows, 1, dim) and three[1].shape == (rows, 1) and torch.equal(three[0][:, 0], y)
    one = features.rms_norm_8bit(x[0].to(DEV), w, res[0].to(DEV), group=64)
    assert one[1].shape == (-(-dim // 64),) and torch.equal(one[0].float(), q[0].float()) and torch.equal(one[1], scale[0])
    flat = features.rms_norm(x.to(DEV), w, res[:1].to(DEV).expand(rows, dim))
    assert torch.equal(flat[2].cpu(), to.stream(x, res[:1]))
    fo.close(flat[0], to.rms_norm(to.stream(x, res[:1]), w.cpu(), EPS)[0], "y")

    want = features.rms_norm_grad(dy.to(DEV), h, rstd, w, more.to(DEV))
    for k in range(4):
        views = [_strided(dy, 3, 3), _strided(h.cpu(), 5, 2), _strided(more, 1, 7), _strided(x, 2, 1)]
        got = features.rms_norm_grad(views[0], views[1], rstd, w, views[2], out=views[k])
        assert got[0] is views[k] and all(_untouched(v) for v in views) and torch.equal(views[k], want[0]) and torch.equal(got[1], want[1])
    flat = features.rms_norm_grad(dy[:1].to(DEV).expand(rows, dim), h, rstd, w)
    for a, b, what in zip(flat, to.rms_norm_grad(dy[:1].expand(rows, dim), h.cpu(), rstd.cpu(), w.cpu(), None, BF16, BF16), ("dh", "dw")):
        fo.close(a, b, what)


# The row's last vector, which begins early, is in another wave than the vector whose columns it overlaps.
@pytest.mark.parametrize("x,dim", [(BF16, 2049), (BF16, 2563), (BF16, 4097), (BF16, 12_289), (F32, 1025), (F32, 2050), (F32, 5123), (F32, 16_129)], ids=str)
def test_rms_norm_in_place_with_the_last_vector_in_another_wave(x, dim):
    g, rows = _gen(dim), 301
    a, res, dy, more = (_rows_of_sizes(g, rows, dim, x).to(DEV) for _ in range(4))
    w = (1 + _normal(g, dim, std=0.3)).to(x).to(DEV)
    y, rstd, h = features.rms_norm(a, w, res)
    q, scale, _, _ = features.rms_norm_8bit(a, w, res)
    dh, dw = features.rms_norm_grad(dy, h, rstd, w, more)
    for out, total in ((0, 1), (1, 0)):
        place = [a.clone(), res.clone()]
        got = features.rms_norm(place[0], w, place[1], out=place[out], sum_out=place[total])
        assert torch.equal(place[out], y) and torch.equal(place[total], h) and torch.equal(got[1], rstd)
    for k in (0, 1):
        place = [a.clone(), res.clone()]
        got = features.rms_norm_8bit(place[0], w, place[1], sum_out=place[k])
        assert torch.equal(got[0].float(), q.float()) and torch.equal(got[1], scale) and torch.equal(place[k], h)
    for k in range(3):
        place = [dy.clone(), h.clone(), more.clone()]
        got = features.rms_norm_grad(place[0], place[1], rstd, w, place[2], out=place[k])
        assert torch.equal(place[k], dh) and torch.equal(got[1], dw)


def test_rms_norm_hard_rows():
    # Zeros, rows far from one and rows that hold an infinity or a NaN, which do not touch the others.
    g = _gen(3)
    dim = 96
    x = torch.stack([torch.zeros(dim), 1e-18 * torch.randn(dim, generator=g), 1e15 * torch.randn(dim, generator=g), torch.randn(dim, generator=g),
                     torch.randn(dim, generator=g), torch.full((dim,), -5.0)])
    y, rstd, _ = features.rms_norm(x.to(DEV))
    want_y, want_rstd = to.rms_norm(x, None, EPS)
    fo.close(y, want_y, "y")
    fo.close(rstd, want_rstd, "rstd")
    for group in (None, 32):
        q, scale, _, _ = features.rms_norm_8bit(x.to(DEV), group=group)
        want_q, want_scale = to.rms_norm_8bit(x, None, EPS, group)
        fo.close(scale, want_scale, "scale")
        _close8(q, want_q, "q")
        assert not q[0].float().any() and (scale[0] == to.TINY).all()
        bad = x.clone()
        bad[0, 3], bad[3, 7], bad[4, 40] = float("inf"), float("nan"), float("inf")
        qb, sb, rb, _ = features.rms_norm_8bit(bad.to(DEV), group=group)
        assert torch.isnan(qb[3].float()).all() and torch.isnan(qb[0, 3].float()) and torch.isnan(qb[4, 40].float())
        assert not qb[4].float().nan_to_num(0.0).any()
        for r in (1, 2, 5):
            assert torch.equal(qb[r].float(), q[r].float()) and torch.equal(sb[r], scale[r]) and rb[r] == rstd[r]
        # an infinite result leaves the other groups as they are
        w = torch.ones(dim)
        w[70] = float("inf")
        qw, sw, _, _ = features.rms_norm_8bit(x.to(DEV), w.to(DEV), group=group)
        assert torch.isinf(sw[3:].view(3, -1)[:, -1]).all() and torch.isnan(qw[3:, 70].float()).all()
        if group:
            assert torch.equal(sw[3:, :2], scale[3:, :2]) and torch.equal(qw[3:, :64].float(), q[3:, :64].float())
    half = torch.full((2, dim), 60_000.0, dtype=F16)  # the sum is beyond the type
    _, _, h = features.rms_norm(half.to(DEV), None, half.to(DEV))
    assert torch.isinf(h).all()


def test_rms_norm_without_rows():
    x, w = torch.empty(0, 33, device=DEV), torch.ones(33, device=DEV)
    y, rstd, h = features.rms_norm(x, w, x)
    assert y.shape == h.shape == (0, 33) and rstd.shape == (0,)
    q, scale, _, _ = features.rms_norm_8bit(x, w, group=32)
    assert q.shape == (0, 33) and scale.shape == (0, 2)
    dh, dw = features.rms_norm_grad(x, x, rstd, w)
    assert dh.shape == (0, 33) and dw.shape == (33,) and not dw.any()
    assert features.rms_norm_grad(x, x, rstd, w, params=False)[1] is None


# Outputs past the caches, wide types and narrow, on the GPU in 64 bits.
@pytest.mark.parametrize("dtype,rows,dim", [(F32, 20_005, 901), (BF16, 40_001, 901), (F16, 7_001, 5_001), (F32, 1_100, 16_001), (BF16, 56_003, 901), (F32, 28_001, 901)])
def test_rms_norm_past_the_caches(dtype, rows, dim):
    g = torch.Generator(device=DEV).manual_seed(rows)
    x, res, dy = (torch.randn(rows, dim, generator=g, device=DEV).to(dtype) for _ in range(3))
    w = (1 + 0.2 * torch.randn(dim, generator=g, device=DEV))
    y, rstd, h = features.rms_norm(x, w, res)
    q, scale, _, h8 = features.rms_norm_8bit(x, w, res, group=128)
    dh, dw = features.rms_norm_grad(dy, h, rstd, w, res)
    assert torch.equal(h, (x.float() + res.float()).to(dtype)) and torch.equal(h8, h)
    for part in range(0, rows, 5_000):
        rows_ = slice(part, min(part + 5_000, rows))
        hd = h[rows_].double()
        r64 = (hd.square().mean(1, keepdim=True) + EPS).rsqrt()
        want = hd * r64 * w.double()
        # rstd is off by (dim's sum's depth / 2 + 6) u at most, the product by 3 u, the rounding by its half step
        u = ((to.depth(dim) + 4) / 2 + 7) * 1.05 * fo.U
        half = fo.ROUND[dtype][0]
        assert ((y[rows_].double() - want).abs() <= (u + 1.05 * half) * want.abs() + 2.0 ** -25).all()
        top = torch.nn.functional.pad(want, (0, -dim % 128)).view(want.shape[0], -1, 128).abs().amax(2) / to.TOP
        assert ((scale[rows_].double() - top).abs() <= (u + 3 * fo.U) * top).all()
        z = want / top.repeat_interleave(128, 1)[:, :dim]
        assert ((q[rows_].float().double() - z).abs() <= to.grid(z) / 2 + (2 * u + 6 * fo.U) * z.abs()).all()
        n, gw = hd * rstd[rows_].double()[:, None], dy[rows_].double() * w.double()
        c = (gw * n).mean(1, keepdim=True)
        want = rstd[rows_].double()[:, None] * (gw - n * c) + res[rows_].double()
        size = rstd[rows_].double()[:, None] * (n.abs() * (to.depth(dim) + 5) * (gw * n).abs().mean(1, keepdim=True) + 5 * (gw.abs() + (n * c).abs())) + want.abs()
        assert ((dh[rows_].double() - want).abs() <= 1.05 * fo.U * size + 1.05 * half * want.abs() + 2.0 ** -25).all()
    n = h.double() * rstd.double()[:, None]
    want, size = (dy.double() * n).sum(0), (dy.double() * n).abs().sum(0)
    # a lane's share of the rows, the groups' and the workgroups' sums: no term takes part in more additions than there are rows
    assert ((dw.double() - want).abs() <= 1.05 * (rows / 64 + 64) * fo.U * size).all()


def test_rms_norm_gradient_against_differences():
    g = _gen(35)
    rows, dim, step = 6, 50, 1e-5
    x, res, dy = (_rows_of_sizes(g, rows, dim, F32) for _ in range(3))
    w = 1 + _normal(g, dim, std=0.3)
    _, rstd, h = features.rms_norm(x.to(DEV), w.to(DEV), res.to(DEV))
    dh, dw = (t.double().cpu() for t in features.rms_norm_grad(dy.to(DEV), h, rstd, w.to(DEV), dy.to(DEV)))

    def loss(h, w):
        y = h * (h.square().mean(1, keepdim=True) + EPS).rsqrt() * w
        return float(((y + h) * dy.double()).sum())

    h0, w0 = h.double().cpu(), w.double()
    for k, grad in enumerate((dh, dw)):
        for _ in range(4):
            way = torch.randn(*grad.shape, generator=g, dtype=torch.float64)
            up, down = [h0, w0], [h0, w0]
            up[k], down[k] = up[k] + step * way, down[k] - step * way
            slope = (loss(*up) - loss(*down)) / (2 * step)
            # the gradient's elements are off by some 1e-6 of their size in 32 bits, and the difference by about
            # step^2 of the loss's third derivative and 1e-16 / step of the loss
            size = float((grad.abs() * way.abs()).sum()) + float(dy.abs().sum())
            assert abs(float((grad * way).sum() - slope)) <= 2e-6 * size, k


def test_rms_norm_offsets_beyond_32_bits():
    rows, dim = 70_000, 32_000  # 2.2e9 elements
    x = torch.zeros(rows, dim, dtype=BF16, device=DEV)
    x[rows - 1] = 3.0
    x[1] = -2.0
    q, scale, rstd, h = features.rms_norm_8bit(x, eps=0.25, group=128)
    assert h is x and (q[rows - 1].float() == to.TOP).all() and (q[1].float() == -to.TOP).all() and not q[rows - 2].float().any()
    assert abs(float(scale[rows - 1, 0]) * to.TOP * (9.25 ** 0.5) / 3 - 1) < 1e-5 and float(rstd[0]) == 2.0
    features.rms_norm(x, eps=0.25, out=x)
    # 3 / sqrt(9.25) = 0.98639 and 2 / sqrt(4.25) = 0.97014, whose nearest in 8 bits of mantissa are 253 / 256 and 248 / 256
    assert (x[rows - 1] == 0.98828125).all() and (x[1] == -0.96875).all() and not x[rows - 2].any() and not x[0].any()


# ---------------------------------------------------------------- refusals


def test_rms_refusals():
    x = torch.randn(6, 64, device=DEV)
    w = torch.ones(64, device=DEV)
    stats = torch.ones(6, device=DEV)
    wide = torch.randn(6, 200, device=DEV)
    q = torch.zeros(6, 64, device=DEV).to(torch.float8_e4m3fn)
    leaf = torch.zeros(6, 64, device=DEV, requires_grad=True)
    bad = [
        lambda: features.rms_norm(x.double()), lambda: features.rms_norm(x.cpu()), lambda: features.rms_norm(x.t()), lambda: features.rms_norm(x[0, 0]),
        lambda: features.rms_norm(x, w[:7]), lambda: features.rms_norm(x, w.cpu()), lambda: features.rms_norm(x, w, x[:5]), lambda: features.rms_norm(x, w, x.half()),
        lambda: features.rms_norm(x, w, x.cpu()), lambda: features.rms_norm(x, out=x.half()), lambda: features.rms_norm(x, sum_out=x.clone()),
        lambda: features.rms_norm(x, w, x, out=wide[:, :64], sum_out=wide[:, :64]), lambda: features.rms_norm(x, w, x, out=wide[:, :64], sum_out=wide[:, 63:127]),
        lambda: features.rms_norm(wide[:, :64], out=wide[:, 1:65]), lambda: features.rms_norm(wide[:, :64], w, wide[:, 64:128], out=wide[:, 32:96]),
        lambda: features.rms_norm(wide[:, :64], w, x, sum_out=wide[:, 8:72]), lambda: features.rms_norm(x, x[2], out=x), lambda: features.rms_norm(x, w, x, sum_out=leaf),
        lambda: features.rms_norm(x, out=leaf), lambda: features.rms_norm_8bit(x, out=x), lambda: features.rms_norm_8bit(x, group=16), lambda: features.rms_norm_8bit(x, group=0),
        lambda: features.rms_norm_8bit(x, out=q[:5]), lambda: features.rms_norm_8bit(x, out=q.t().contiguous().t()),
        lambda: features.rms_norm_8bit(x, out=x.view(torch.float8_e4m3fn)[:, :64]),
        lambda: features.rms_norm_grad(x.half(), x, stats), lambda: features.rms_norm_grad(x, x, stats[:5]), lambda: features.rms_norm_grad(x, x, stats.double()),
        lambda: features.rms_norm_grad(x, x, stats, w, x[:5]), lambda: features.rms_norm_grad(x, x, stats, w[:5]),
        lambda: features.rms_norm_grad(wide[:, :64], x, stats, w, out=wide[:, 4:68]), lambda: features.rms_norm_grad(x, wide[:, :64], stats, w, out=wide[:, 4:68]),
        lambda: features.rms_norm_grad(x, x, stats, w, wide[:, :64], out=wide[:, 4:68]), lambda: features.rms_norm_grad(x, x, wide.view(-1)[3:9], w, out=wide[:, :64]),
    ]
    for k, f in enumerate(bad):
        with pytest.raises(ValueError):
            print("refusal", k)
            f()
    for f in (lambda: features.rms_norm(x, torch.ones(64, device=DEV).half()), lambda: features.rms_norm(x, eps=-1.0),
              lambda: features.rms_norm_grad(x, x, stats, torch.ones(64, device=DEV).half())):
        with pytest.raises(scd.ScdError):
            f()
    # side by side in one buffer they share nothing
    before = wide[:, :64].clone()
    y, _, h = features.rms_norm(wide[:, :64], w, x, out=wide[:, 64:128], sum_out=wide[:, 128:192])
    assert torch.equal(wide[:, :64], before) and torch.equal(h, before + x) and torch.equal(y, features.rms_norm(before, w, x)[0])


def test_rms_writes_count_as_in_place_operations():
    x, w, stats = torch.randn(6, 64, device=DEV), torch.ones(64, device=DEV), torch.ones(6, device=DEV)
    y, total, q = torch.empty_like(x), torch.empty_like(x), torch.empty(6, 64, device=DEV).to(torch.float8_e4m3fn)
    before = [t._version for t in (x, y, total, q)]
    features.rms_norm(x, w, x, out=y, sum_out=total)
    features.rms_norm_8bit(x, w, out=q)
    features.rms_norm_grad(x, x, stats, w, out=y)
    assert [t._version - b for t, b in zip((x, y, total, q), before)] == [0, 2, 1, 1]


# A width for every group of lanes and every type: matrices that go past the caches are copies of a small one, each of which
# has to lie within the small one's bounds.
@pytest.mark.parametrize("x,p", PAIRS)
@pytest.mark.parametrize("dim", [3, 14, 30, 60, 120, 250, 500, 700, 1000, 1500, 2000, 2500, 4000, 5000, 6000, 7000, 8000, 10_000, 12_000, 16_000])
def test_rms_norm_widths_past_the_caches(dim, x, p):
    g = torch.Generator(device=DEV).manual_seed(dim)
    few = 37
    small = [torch.randn(few, dim, generator=g, device=DEV).to(x) for _ in range(3)]
    w = (1 + 0.3 * torch.randn(dim, generator=g, device=DEV)).to(p)
    copies = -(-int(1.03 * (384 << 20)) // (few * dim * small[0].element_size() * 3))  # of three matrices; four and more are above every limit
    big = [t.repeat(copies, 1) for t in small]

    def within(got, want, what):
        value, bound = (t.to(DEV) for t in want)
        got = got.view(-1, *value.shape)
        for part in got.split(max(1, 30_000_000 // value.numel())):
            bad = (part.double() - value).abs() > bound
            assert not bad.any(), f"{what}: {int(bad.sum())} of {part.numel()} outside their bound"

    host = [t.cpu() for t in small]
    for res in (False, True):
        xs = big[0] if res else big[0].repeat(2, 1)  # without a residual, two matrices: twice the rows
        h = to.stream(host[0], host[1] if res else None)
        want_y, want_rstd = to.rms_norm(h, w.cpu(), EPS)
        y, rstd, kept = features.rms_norm(xs, w, big[1] if res else None)
        within(y, want_y, "y")
        within(rstd, want_rstd, "rstd")
        assert torch.equal(kept.view(-1, few, dim), h.to(DEV).expand(kept.shape[0] // few, few, dim))
        del y
        for group in (None, 64):
            q, scale, _, _ = features.rms_norm_8bit(xs, w, big[1] if res else None, group=group)
            want_q, want_scale = to.rms_norm_8bit(h, w.cpu(), EPS, group)
            within(q.float(), want_q, f"q {group}")
            within(scale, want_scale, f"scale {group}")
            del q
    _, rstd, _ = features.rms_norm(small[0], w)
    for res in (False, True):
        dh, dw = features.rms_norm_grad(big[2], big[0], rstd.repeat(copies), w, big[1] if res else None)
        want_dh, _ = to.rms_norm_grad(host[2], host[0], rstd.cpu(), w.cpu(), host[1] if res else None, x, p)
        within(dh, want_dh, "dh")
        terms = small[2].double() * (small[0].double() * rstd.double()[:, None])
        # no term takes part in more additions than a lane has rows, and the groups' and workgroups' sums
        bound = copies * terms.abs().sum(0) * (few * copies / 256 + 64) * 1.05 * fo.U + (1.05 * fo.ROUND[p][0]) * copies * terms.sum(0).abs() + 2.0 ** -24
        value, largest = copies * terms.sum(0), torch.finfo(p).max
        over = value.abs() - bound > largest  # sums of 600,000 rows may be beyond fp16: infinite
        assert torch.equal(torch.isinf(dw), over) and torch.equal(torch.sign(dw)[over], torch.sign(value)[over].to(p))
        assert ((dw.double() - value).abs() <= bound)[~over].all()
