"""The operators of learned features on the GPU against their 64-bit oracle (tests/_features_oracle.py, whose
bounds come from the operations' roundings), at the sizes, masks, strides and types where they can go wrong."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import _features_oracle as fo  # noqa: E402
from paper_1702_07005_amd import features, scd  # noqa: E402

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
PAIRS = [(a, b) for a in TYPES for b in TYPES]


@pytest.fixture(scope="module", autouse=True)
def _give_back_memory():
    yield
    torch.cuda.empty_cache()


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _normal(g, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(*shape, generator=g) * std).to(dtype)


def _strided(t, pad, offset=0):
    """A device copy whose rows lie `pad` elements further apart and begin `offset` elements into the memory."""
    n, d = t.shape
    room = torch.full((offset + n * (d + pad) + 8,), float("nan"), dtype=t.dtype, device=DEV)
    v = room[offset:offset + n * (d + pad)].view(n, d + pad)[:, :d]
    v.copy_(t)
    return v


def _untouched(v):
    """The elements between the rows of a view made by `_strided` are still NaN."""
    n, d = v.shape
    whole = v.as_strided((n, v.stride(0)), (v.stride(0), 1), v.storage_offset())
    return bool(torch.isnan(whole[:, d:]).all())


# ---------------------------------------------------------------- lookup


@pytest.mark.parametrize("table,out", PAIRS)
@pytest.mark.parametrize("n,dim", [(1, 1), (1, 4096), (3, 7), (130, 33), (67, 300)])
def test_embed(table, out, n, dim):
    g = _gen(n * 10_000 + dim)
    rows = 57
    e = _normal(g, rows, dim, dtype=TYPES[table])
    t = torch.randint(0, rows, (n,), generator=g)
    t[n // 2] = rows - 1
    got = features.embed(t.to(DEV), e.to(DEV), scale=3.7, dtype=TYPES[out])
    assert got.dtype == TYPES[out] and got.shape == (n, dim)
    fo.close(got, fo.embed(t, e, float(torch.tensor(3.7)), TYPES[out]), "embed")


@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
def test_embed_outside_tokens_views_and_shapes(ids):
    g = _gen(11)
    rows, dim = 40, 25
    e = _normal(g, rows, dim, dtype=torch.bfloat16)
    t = torch.randint(-3, rows + 3, (5, 6, 7), generator=g).to(ids)
    ev = _strided(e, 9, offset=3)
    out = torch.full((5 * 6 * 7, dim + 4), float("inf"), device=DEV)
    o = out[:, :dim].view(5, 6, 7, dim)
    got = features.embed(t.to(DEV), ev, scale=-0.5, out=o)
    assert got is o
    fo.close(got, fo.embed(t, e, -0.5, torch.float32), "embed")
    assert torch.isinf(out[:, dim:]).all()
    if ids == torch.int64:  # tokens whose low 32 bits alone would name a row
        far = torch.tensor([1 << 32, (1 << 32) + 5, -(1 << 32), 5], device=DEV)
        got = features.embed(far, ev)
        assert torch.isnan(got[:2]).all() and not got[2].any() and torch.equal(got[3], ev[5])


def test_embed_many_rows_in_flight_and_none():
    g = _gen(12)
    e = _normal(g, 1000, 16)
    t = torch.randint(-1, 1000, (70_001,), generator=g)
    got = features.embed(t.to(DEV), e.to(DEV))
    fo.close(got, fo.embed(t, e, 1.0, torch.float32), "embed")
    assert features.embed(t[:0].to(DEV), e.to(DEV)).shape == (0, 16)
    assert torch.isnan(features.embed(t[:3].abs().to(DEV), e[:0].to(DEV))).all()
    masked = e.clone()
    masked[0] = float("nan")  # row 0 does not leak into padded places
    assert not features.embed(torch.full((9,), -1, device=DEV), masked.to(DEV)).any()


def test_embed_table_above_32_bit_offsets():
    rows, dim = 40_000, 65_536  # 2.6e9 elements
    e = torch.zeros(rows, dim, dtype=torch.bfloat16, device=DEV)
    e[rows - 1] = 2.0
    e[1] = 3.0
    got = features.embed(torch.tensor([rows - 1, 1, 0], device=DEV), e)
    assert (got[0] == 2).all() and (got[1] == 3).all() and not got[2].any()
    grad = torch.ones(2, dim, dtype=torch.bfloat16, device=DEV)
    features.embed_grad(torch.tensor([rows - 1, 2], device=DEV), grad, rows, out=e)
    assert (e[rows - 1] == 1).all() and (e[2] == 1).all() and not e[1].any() and not e[rows - 2].any()


# ---------------------------------------------------------------- its gradient


def _tokens(g, n, rows, kind):
    if kind == "even":
        return torch.randint(0, rows, (n,), generator=g)
    if kind == "zipf":
        u = torch.rand(n, generator=g, dtype=torch.float64)
        return (torch.exp(u * torch.log(torch.tensor(rows + 1.0))) - 1).long().clamp(0, rows - 1)
    if kind == "one":
        return torch.full((n,), rows - 1)
    if kind == "none":
        return torch.full((n,), -1)
    t = torch.randint(-2, rows + 2, (n,), generator=g)  # "outside": some of either side
    return t


@pytest.mark.parametrize("grad,out", PAIRS)
@pytest.mark.parametrize("n,rows,dim", [(1, 1, 1), (9, 5, 7), (300, 1000, 33), (777, 41, 300)])
def test_embed_grad_types(grad, out, n, rows, dim):
    g = _gen(n + rows + dim)
    t = _tokens(g, n, rows, "zipf")
    d = _normal(g, n, dim, dtype=TYPES[grad])
    got = features.embed_grad(t.to(DEV), d.to(DEV), rows, scale=1.5, dtype=TYPES[out])
    fo.close(got, fo.embed_grad(t, d, rows, 1.5, TYPES[out]), "embed_grad")


# Around the sorts' limits: one launch up to 1,024 tokens, tiles up to 16,384 or, where a key has several digits, 32,768,
# and the radix sort with two entries a thread in one and two passes.
@pytest.mark.parametrize("kind", ["even", "zipf", "one", "none", "outside"])
@pytest.mark.parametrize("n,rows,dim", [(64, 3, 16), (1023, 300, 5), (1024, 70_000, 8), (1025, 513, 8), (4096, 511, 9), (4097, 512, 4),
                                        (16_384, 1025, 8), (16_385, 7, 8), (16_390, 2047, 6), (40_001, 2048, 8), (50_000, 300_000, 3),
                                        (20_000, 5_000_000, 2)])
def test_embed_grad_sorts(kind, n, rows, dim):
    g = _gen(n + rows)
    t = _tokens(g, n, rows, kind)
    d = _normal(g, n, dim)
    got = features.embed_grad(t.to(DEV), d.to(DEV), rows)
    fo.close(got, fo.embed_grad(t, d, rows, 1.0, torch.float32), f"embed_grad {kind}")


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n,rows,dim", [(500, 90, 31), (18_000, 333, 20), (6, 4, 2100)])
def test_embed_grad_views_and_accumulation(accumulate, n, rows, dim):
    g = _gen(n + dim)
    t = _tokens(g, n, rows, "outside")
    d = _normal(g, n, dim, dtype=torch.float16)
    before = _normal(g, rows, dim, dtype=torch.bfloat16)
    out = _strided(before, 5, offset=1)
    got = features.embed_grad(t.int().to(DEV), _strided(d, 3, offset=7), rows, scale=2.0, out=out, accumulate=accumulate)
    assert got is out and _untouched(out)
    fo.close(got, fo.embed_grad(t, d, rows, 2.0, torch.bfloat16, before if accumulate else None), "embed_grad")


def test_embed_grad_rows_left_alone_and_broadcast_gradients():
    g = _gen(31)
    before = torch.full((50, 12), float("inf"), device=DEV)
    t = torch.tensor([3, 3, 7], device=DEV)
    one = _normal(g, 1, 12)
    got = features.embed_grad(t, one.to(DEV).expand(3, 12), 50, out=before, accumulate=True)
    assert torch.isinf(got).all()
    got = features.embed_grad(t, one.to(DEV).expand(3, 12), 50)
    fo.close(got, fo.embed_grad(t.cpu(), one.expand(3, 12), 50, 1.0, torch.float32), "embed_grad")
    # gradients of padded places may hold anything
    d = _normal(g, 4, 12)
    d[1] = float("nan")
    got = features.embed_grad(torch.tensor([0, -1, 50, 0], device=DEV)[:2], d[:2].to(DEV), 50)
    fo.close(got, fo.embed_grad(torch.tensor([0, -1]), d[:2], 50, 1.0, torch.float32), "embed_grad")
    empty = features.embed_grad(t[:0], one[:0].to(DEV), 50, out=before)
    assert not empty.any()
    assert features.embed_grad(t, one.to(DEV).expand(3, 12), 0).shape == (0, 12)


def test_embed_grad_is_the_same_every_time():
    g = _gen(33)
    t = _tokens(g, 60_000, 900, "zipf").to(DEV)
    d = _normal(g, 60_000, 40).to(DEV)
    first = features.embed_grad(t, d, 900)
    for _ in range(3):
        assert torch.equal(features.embed_grad(t, d, 900), first)


def test_embed_gradient_against_differences():
    # The lookup is linear in its table: a difference along any direction is the derivative.
    g = _gen(34)
    rows, dim, n = 30, 17, 200
    t = _tokens(g, n, rows, "outside").clamp(max=rows - 1)
    d = _normal(g, n, dim)
    grad = features.embed_grad(t.to(DEV), d.to(DEV), rows, scale=1.25).double().cpu()
    _, bound = fo.embed_grad(t, d, rows, 1.25, torch.float32)
    for _ in range(4):
        way = torch.randn(rows, dim, generator=g, dtype=torch.float64)
        slope = (fo.embed(t, way, 1.25, torch.float32)[0] * d.double()).sum()
        assert abs(float((grad * way).sum() - slope)) <= float((bound * way.abs()).sum()) + 1e-12 * n * dim


# ---------------------------------------------------------------- layer norm


DIMS = [1, 3, 7, 8, 9, 31, 64, 65, 127, 200, 256, 257, 511, 777, 1024, 1030, 2049, 4096, 4100, 8192, 8193, 16_384, 16_391, 40_000]


def _features_like(g, rows, dim, dtype):
    x = _normal(g, rows, dim) * (0.1 + 2 * torch.rand(rows, 1, generator=g)) + 0.4
    return x.to(dtype)


@pytest.mark.parametrize("x,p", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("dim", DIMS)
def test_layer_norm_and_gradient(x, p, dim):
    g = _gen(dim)
    rows = 5 if dim > 2000 else 37
    xt, pt = TYPES[x], TYPES[p]
    xs = _features_like(g, rows, dim, xt)
    w, b = (1 + _normal(g, dim, std=0.3)).to(pt), _normal(g, dim, dtype=pt)
    y, mean, rstd = features.layer_norm(xs.to(DEV), w.to(DEV), b.to(DEV), eps=1e-5)
    want = fo.layer_norm(xs, w, b, float(torch.tensor(1e-5)), xt)
    for got, v, what in zip((y, mean, rstd), want, ("y", "mean", "rstd")):
        fo.close(got, v, f"layer_norm {what}")
    dy = _normal(g, rows, dim, dtype=xt)
    grads = features.layer_norm_grad(dy.to(DEV), xs.to(DEV), mean, rstd, w.to(DEV))
    want = fo.layer_norm_grad(dy, xs, mean.cpu(), rstd.cpu(), w, xt, pt)
    for got, v, what in zip(grads, want, ("x", "weight", "bias")):
        fo.close(got, v, f"layer_norm_grad {what}")


@pytest.mark.parametrize("rows,dim", [(1, 64), (2, 4096), (255, 16), (2049, 24), (5003, 40), (3001, 300), (700, 1500), (9001, 5)])
def test_layer_norm_rows(rows, dim):
    g = _gen(rows + dim)
    xs, w, b = _features_like(g, rows, dim, torch.float32), 1 + _normal(g, dim, std=0.3), _normal(g, dim)
    y, mean, rstd = features.layer_norm(xs.to(DEV), w.to(DEV), b.to(DEV))
    for got, v in zip((y, mean, rstd), fo.layer_norm(xs, w, b, float(torch.tensor(1e-5)), torch.float32)):
        fo.close(got, v, "layer_norm")
    dy = _normal(g, rows, dim)
    grads = features.layer_norm_grad(dy.to(DEV), xs.to(DEV), mean, rstd, w.to(DEV))
    for got, v in zip(grads, fo.layer_norm_grad(dy, xs, mean.cpu(), rstd.cpu(), w, torch.float32, torch.float32)):
        fo.close(got, v, "layer_norm_grad")
    again = features.layer_norm_grad(dy.to(DEV), xs.to(DEV), mean, rstd, w.to(DEV))
    assert all(torch.equal(a, b) for a, b in zip(grads, again))


@pytest.mark.parametrize("dim", [20, 513, 17_000])
def test_layer_norm_views_in_place_and_without_parameters(dim):
    g = _gen(dim)
    rows = 11
    xs = _features_like(g, rows, dim, torch.bfloat16)
    dy = _normal(g, rows, dim, dtype=torch.bfloat16)
    plain = features.layer_norm(xs.to(DEV))
    for got, v in zip(plain, fo.layer_norm(xs, None, None, float(torch.tensor(1e-5)), torch.bfloat16)):
        fo.close(got, v, "layer_norm")
    xv, yv = _strided(xs, 7, offset=1), _strided(xs, 3, offset=5)
    got = features.layer_norm(xv, out=yv)
    assert got[0] is yv and _untouched(yv) and torch.equal(yv, plain[0]) and torch.equal(got[1], plain[1])
    same = features.layer_norm(xv, out=xv)
    assert same[0] is xv and _untouched(xv) and torch.equal(xv, plain[0])
    three = features.layer_norm(xs.to(DEV).view(rows, 1, dim))
    assert three[0].shape == (rows, 1, dim) and three[1].shape == (rows, 1) and torch.equal(three[0][:, 0], plain[0])
    one = features.layer_norm(xs[0].to(DEV))
    assert one[1].shape == () and torch.equal(one[0], plain[0][0])

    _, mean, rstd = plain
    want = fo.layer_norm_grad(dy, xs, mean.cpu(), rstd.cpu(), None, torch.bfloat16, torch.bfloat16)
    grads = features.layer_norm_grad(dy.to(DEV), xs.to(DEV), mean, rstd)
    for got, v in zip(grads, want):
        fo.close(got, v, "layer_norm_grad")
    dx, dw, db = features.layer_norm_grad(dy.to(DEV), xs.to(DEV), mean, rstd, params=False)
    assert dw is None and db is None and torch.equal(dx, grads[0])
    gv, xv = _strided(dy, 3, offset=3), _strided(xs, 5, offset=2)
    out = _strided(xs, 1, offset=9)
    into = features.layer_norm_grad(gv, xv, mean, rstd, out=out)
    assert into[0] is out and _untouched(out) and all(torch.equal(a, b) for a, b in zip(into, grads))
    over = features.layer_norm_grad(gv, xv, mean, rstd, out=gv)
    assert _untouched(gv) and torch.equal(over[0], grads[0]) and torch.equal(over[1], grads[1])
    over = features.layer_norm_grad(dy.to(DEV), xv, mean, rstd, out=xv)
    assert _untouched(xv) and torch.equal(over[0], grads[0]) and torch.equal(over[2], grads[2])
    # one gradient for all rows
    flat = features.layer_norm_grad(dy[:1].to(DEV).expand(rows, dim), xs.to(DEV), mean, rstd)
    for got, v in zip(flat, fo.layer_norm_grad(dy[:1].expand(rows, dim), xs, mean.cpu(), rstd.cpu(), None, torch.bfloat16, torch.bfloat16)):
        fo.close(got, v, "layer_norm_grad")


def test_layer_norm_hard_rows():
    # A constant row has zero variance, a row far from zero loses nothing to its mean, and a row that holds an infinity
    # or a NaN does not touch the others.
    g = _gen(3)
    dim = 96
    xs = torch.stack([torch.full((dim,), 5.0), 1000 + torch.randn(dim, generator=g), torch.zeros(dim), 1e-18 * torch.randn(dim, generator=g),
                      1e15 * torch.randn(dim, generator=g), torch.randn(dim, generator=g), torch.randn(dim, generator=g)])
    y, mean, rstd = features.layer_norm(xs.to(DEV))
    for got, v in zip((y, mean, rstd), fo.layer_norm(xs, None, None, float(torch.tensor(1e-5)), torch.float32)):
        fo.close(got, v, "layer_norm")
    bad = xs.clone()
    bad[0, 3], bad[5, 7] = float("inf"), float("nan")
    yb, mb, rb = features.layer_norm(bad.to(DEV))
    assert torch.isnan(yb[0]).any() and torch.isnan(yb[5]).all()
    for r in (1, 2, 3, 4, 6):
        assert torch.equal(yb[r], y[r]) and mb[r] == mean[r] and rb[r] == rstd[r]


def test_layer_norm_without_rows():
    x = torch.empty(0, 33, device=DEV)
    w = torch.ones(33, device=DEV)
    y, mean, rstd = features.layer_norm(x, w)
    assert y.shape == (0, 33) and mean.shape == (0,)
    dx, dw, db = features.layer_norm_grad(x, x, mean, rstd, w)
    assert dx.shape == (0, 33) and not dw.any() and not db.any()


def test_layer_norm_gradient_against_differences():
    g = _gen(35)
    rows, dim, h = 6, 50, 1e-5
    xs, w, dy = _features_like(g, rows, dim, torch.float32), 1 + _normal(g, dim, std=0.3), _normal(g, rows, dim)
    b = torch.zeros(dim)
    _, mean, rstd = features.layer_norm(xs.to(DEV), w.to(DEV), b.to(DEV))
    grads = [t.double().cpu() for t in features.layer_norm_grad(dy.to(DEV), xs.to(DEV), mean, rstd, w.to(DEV))]

    def loss(x, w, b):
        return float((fo.layer_norm(x, w, b, 1e-5, torch.float32)[0][0] * dy.double()).sum())

    x0, w0, b0 = xs.double(), w.double(), b.double()
    for k, at in enumerate((x0, w0, b0)):
        for _ in range(4):
            way = torch.randn(*at.shape, generator=g, dtype=torch.float64)
            up, down = [x0, w0, b0], [x0, w0, b0]
            up[k], down[k] = at + h * way, at - h * way
            slope = (loss(*up) - loss(*down)) / (2 * h)
            # the gradient's elements are off by some 1e-6 of their size in 32 bits, and the difference by about
            # h^2 of the loss's third derivative and 1e-16 / h of the loss
            size = float((grads[k].abs() * way.abs()).sum()) + float(dy.abs().sum())
            assert abs(float((grads[k] * way).sum()) - slope) <= 2e-6 * size, k


# ---------------------------------------------------------------- clipping


def _tensors(g, dtypes, sizes):
    return [_normal(g, n, dtype=TYPES[dtypes[i % len(dtypes)]], std=0.1) for i, n in enumerate(sizes)]


SIZES = [1, 5, 8191, 8192, 8193, 40_000, 3, 0, 16_384, 777]


@pytest.mark.parametrize("dtypes", [("f32",), ("bf16",), ("f16",), ("f32", "bf16", "f16")])
@pytest.mark.parametrize("limit", [1e-3, 1.0, 1e6, float("inf")])
def test_clip(dtypes, limit):
    g = _gen(len(dtypes))
    cpu = _tensors(g, dtypes, SIZES)
    for wide in (False, True):
        dev = [t.to(DEV) for t in cpu]
        outs = [torch.full_like(t, float("nan"), dtype=torch.float32 if wide else t.dtype) for t in dev]
        norm = features.clip_grads(dev, limit, out=outs)
        want_norm, want = fo.clip(cpu, float(torch.tensor(limit)), [o.dtype for o in outs])
        assert norm.shape == () and norm.dtype == torch.float32
        fo.close(norm, want_norm, "norm")
        for a, b, v in zip(dev, cpu, want):
            assert torch.equal(a.cpu(), b)
        for i, (o, v) in enumerate(zip(outs, want)):
            fo.close(o, v, f"clip {i}")
        if not wide:
            same = features.clip_grads(dev, limit)
            assert torch.equal(same, norm) and all(torch.equal(a, b) for a, b in zip(dev, outs))


def test_clip_odd_places_many_tensors_and_norm():
    g = _gen(8)
    flat = _normal(g, 30_000, dtype=torch.bfloat16)
    sizes = [1 + (i * 37) % 211 for i in range(250)]  # several launches
    dev, at, cpu = flat.to(DEV), 1, []
    parts = []
    for n in sizes:
        parts.append(dev[at:at + n])
        cpu.append(flat[at:at + n])
        at += n
    norm = features.grad_norm(parts)
    want_norm, want = fo.clip(cpu, 2.0, [torch.bfloat16] * len(cpu))
    fo.close(norm, want_norm, "norm")
    assert torch.equal(dev.cpu(), flat)
    assert torch.equal(features.clip_grads(parts, 2.0), norm)
    for p, v in zip(parts, want):
        fo.close(p, v, "clip")
    assert torch.equal(dev[at:].cpu(), flat[at:]) and torch.equal(dev[:1].cpu(), flat[:1])


def test_clip_extremes():
    big = torch.full((5000,), 3e37, device=DEV)  # squares beyond 32 bits
    out = torch.empty_like(big)
    norm = features.clip_grads([big], 1.0, out=[out])
    want = 3e37 * 5000 ** 0.5
    assert torch.isinf(norm) or abs(float(norm) / want - 1) < 1e-6
    assert float((out.double() * 5000 ** 0.5 - 1).abs().max()) < 1e-6
    tiny = torch.full((10,), 1e-30, device=DEV)
    norm = features.clip_grads([tiny], 1.0)
    assert abs(float(norm) / (1e-30 * 10 ** 0.5) - 1) < 1e-6 and (tiny == 1e-30).all()
    for value in (float("nan"), float("inf")):
        a, b = torch.ones(20_000, device=DEV), torch.ones(3, device=DEV)
        a[12_345] = value
        norm = features.clip_grads([a, b], 1.0)
        assert torch.isnan(norm) if value != value else torch.isinf(norm)
        assert torch.isnan(a[12_345])
        assert torch.isnan(b).all() if value != value else not b.any()
    zero = torch.zeros(7, device=DEV)
    assert features.clip_grads([zero], 0.0) == 0 and not zero.any()
    assert features.grad_norm([torch.empty(0, device=DEV)]) == 0


# ---------------------------------------------------------------- streams, graphs, refusals


def _step(ids, table, weight, bias, dy, stream=None):
    x = features.embed(ids, table, scale=4.0, stream=stream)
    y, mean, rstd = features.layer_norm(x, weight, bias, stream=stream)
    dx, dw, db = features.layer_norm_grad(dy, x, mean, rstd, weight, stream=stream)
    dtable = features.embed_grad(ids, dx, table.shape[0], scale=4.0, stream=stream)
    norm = features.clip_grads([dtable, dw, db], 0.5, stream=stream)
    return y, dtable, dw, db, norm


def _step_inputs(seed, n=20_000, rows=700, dim=48):
    g = _gen(seed)
    return (_tokens(g, n, rows, "outside").clamp(max=rows - 1).to(DEV), _normal(g, rows, dim).to(DEV), 1 + _normal(g, dim, std=0.1).to(DEV),
            _normal(g, dim).to(DEV), _normal(g, n, dim).to(DEV))


def test_other_stream():
    inputs = _step_inputs(1)
    want = _step(*inputs)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for given in (side, side.cuda_stream):
        got = _step(*inputs, stream=given)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_graph_replays():
    inputs = _step_inputs(2)
    other = _step_inputs(3)
    static = [t.clone() for t in inputs]
    _step(*static)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _step(*static)
    for source in (inputs, other, inputs, other):
        for a, b in zip(static, source):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        want = _step(*source)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_refusals():
    x = torch.randn(6, 8, device=DEV)
    ids = torch.zeros(6, dtype=torch.int64, device=DEV)
    stats = torch.zeros(6, device=DEV)
    bad = [
        lambda: features.embed(ids.float(), x), lambda: features.embed(ids.cpu(), x), lambda: features.embed(ids[::2], x),
        lambda: features.embed(ids, x.cpu()), lambda: features.embed(ids, x.double()), lambda: features.embed(ids, x.t()),
        lambda: features.embed(ids, x[None]), lambda: features.embed(ids, x, out=torch.empty(5, 8, device=DEV)),
        lambda: features.embed(ids, x, dtype=torch.float64),
        lambda: features.embed_grad(ids, x[:5], 9), lambda: features.embed_grad(ids, x, 9, accumulate=True),
        lambda: features.embed_grad(ids, x.t().contiguous().t(), 9), lambda: features.embed_grad(ids, x, 9, out=x),
        lambda: features.layer_norm(x.double()), lambda: features.layer_norm(x, torch.ones(7, device=DEV)),
        lambda: features.layer_norm(x, torch.ones(8, device=DEV), torch.ones(8, device=DEV).half()),
        lambda: features.layer_norm(x, out=x.half()), lambda: features.layer_norm(x.t()),
        lambda: features.layer_norm_grad(x.half(), x, stats, stats), lambda: features.layer_norm_grad(x, x, stats[:5], stats),
        lambda: features.layer_norm_grad(x, x, stats, stats.double()),
        lambda: features.clip_grads([], 1.0), lambda: features.clip_grads([x.t()], 1.0), lambda: features.clip_grads([x.double()], 1.0),
        lambda: features.clip_grads([x], 1.0, out=[]), lambda: features.clip_grads([x], 1.0, out=[x.half()]),
        lambda: features.clip_grads([x, x.cpu()], 1.0),
    ]
    for k, f in enumerate(bad):
        with pytest.raises(ValueError):
            print("refusal", k)
            f()
    for f in (lambda: features.layer_norm(x, torch.ones(8, device=DEV).half()), lambda: features.layer_norm(x, eps=-1.0),
              lambda: features.clip_grads([x], -1.0), lambda: features.embed_grad(ids, x, -1)):
        with pytest.raises(scd.ScdError):
            f()


# Few tokens take one launch without a sort, up to 1,024 of them; with long runs, wide rows and more rows than one
# workgroup's 16,384.
@pytest.mark.parametrize("kind", ["even", "zipf", "one", "none", "outside"])
@pytest.mark.parametrize("n,rows,dim", [(2, 40_000, 3), (64, 20, 40), (300, 17_000_000, 1), (511, 33, 2050), (512, 700, 130), (513, 700, 130)])
def test_embed_grad_few_tokens(kind, n, rows, dim):
    g = _gen(n + rows + dim)
    t = _tokens(g, n, rows, kind)
    d = _normal(g, n, dim, dtype=torch.bfloat16)
    got = features.embed_grad(t.to(DEV), d.to(DEV), rows, dtype=torch.float32)
    want = fo.embed_grad(t, d, rows, 1.0, torch.float32)
    fo.close(got, want, f"embed_grad {kind}")
    got.fill_(0.5)
    features.embed_grad(t.to(DEV), d.to(DEV), rows, out=got, accumulate=True)
    if rows < 1_000_000:
        fo.close(got, fo.embed_grad(t, d, rows, 1.0, torch.float32, torch.full((rows, dim), 0.5)), f"embed_grad {kind}")


@pytest.mark.parametrize("kind", ["zipf", "one", "outside"])
@pytest.mark.parametrize("n,rows,dim", [(1023, 90, 17), (1024, 2, 260), (1024, 5000, 64), (1025, 5000, 64), (700, 64, 3)])
def test_embed_grad_few_tokens_long_runs(kind, n, rows, dim):
    g = _gen(n + rows + dim)
    t = _tokens(g, n, rows, kind)
    d = _normal(g, n, dim)
    got = features.embed_grad(t.to(DEV), d.to(DEV), rows)
    fo.close(got, fo.embed_grad(t, d, rows, 1.0, torch.float32), f"embed_grad {kind}")


# One workgroup does few rows for each of its groups alone; one row needs no workspace in any case.
@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("rows,dim", [(1, 5), (64, 30), (65, 30), (8, 700), (9, 700), (2, 5000), (3, 5000), (1, 33_000), (2, 33_000), (3, 33_000)])
def test_layer_norm_gradient_of_few_rows(x, rows, dim):
    g = _gen(rows + dim)
    xt = TYPES[x]
    xs, w, dy = _features_like(g, rows, dim, xt), 1 + _normal(g, dim, std=0.3), _normal(g, rows, dim, dtype=xt)
    _, mean, rstd = features.layer_norm(xs.to(DEV), w.to(DEV))
    want = fo.layer_norm_grad(dy, xs, mean.cpu(), rstd.cpu(), w, xt, torch.float32)
    got = features.layer_norm_grad(dy.to(DEV), xs.to(DEV), mean, rstd, w.to(DEV))
    for a, v, what in zip(got, want, ("x", "weight", "bias")):
        fo.close(a, v, f"layer_norm_grad {what}")
    xd = xs.to(DEV)
    over = features.layer_norm_grad(dy.to(DEV), xd, mean, rstd, w.to(DEV), out=xd)
    assert over[0] is xd and all(torch.equal(a, b) for a, b in zip(over, got))


def test_example_trains_the_table_under_the_readout():
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import learned_features
    objectives = learned_features.train(iterations=8, n=4096)
    # the first read-out is fitted on random vectors; training them has to more than halve what it leaves
    assert objectives[-1] < 0.5 * objectives[0], objectives


@pytest.mark.parametrize("n", [1, 40, 1000])
def test_embed_grad_few_tokens_into_a_large_table(n):
    # zeros by pieces of memory: rows of an odd width, in two column ranges, before, between and after the tokens' rows
    g = _gen(n)
    rows, dim = 16_001, 1051
    t = torch.randint(0, rows, (n,), generator=g)
    t[0] = rows - 1
    if n > 2:
        t[1:3] = torch.tensor([0, 1])
    d = _normal(g, n, dim)
    out = torch.full((rows, dim), float("nan"), device=DEV)
    features.embed_grad(t.to(DEV), d.to(DEV), rows, out=out)
    fo.close(out, fo.embed_grad(t, d, rows, 1.0, torch.float32), "embed_grad")
