"""The AdamW step on the GPU against its 64-bit oracle (tests/_training_oracle.py), and whole training steps with it and the
root-mean-square norm: on other streams, captured and replayed, and as an example runs them."""
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
TYPES = [(F32, F32), (F32, BF16), (F32, F16), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)]
BETAS = (0.9, 0.999)


@pytest.fixture(scope="module", autouse=True)
def _give_back_memory():
    yield
    torch.cuda.empty_cache()


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _normal(g, *shape, dtype=F32, std=1.0):
    return (torch.randn(*shape, generator=g) * std).to(dtype)


def _state(g, n, bits, std):
    """A state as some steps leave it."""
    m, r = _normal(g, n, std=0.3 * std), (torch.rand(n, generator=g) + 0.5) * std
    if bits == 32:
        return m, r.square()
    out = []
    for x in (m, r):
        scale = (to.blocks(x).abs().amax(1) / to.TOP).clamp(min=to.TINY)
        q = (to.blocks(x) / scale[:, None]).reshape(-1)[:n].to(torch.float8_e4m3fn)
        out.append((q, scale))
    return out[0][0], out[1][0], out[0][1], out[1][1]


def _odd(t, offset, room=8):
    """A device copy that begins `offset` elements into its memory, with 8 more behind it, all of them ones before."""
    whole = torch.ones(offset + t.numel() + room, device=DEV).to(t.dtype)
    whole[offset:offset + t.numel()].copy_(t.reshape(-1))
    return whole[offset:offset + t.numel()].view(t.shape), whole


def _around(whole, offset, n):
    w = whole.float()
    return bool((w[:offset] == 1).all() and (w[offset + n:] == 1).all())


def _check_step(sizes, p_type, g_type, bits, copy=None, step=7, lr=2e-3, betas=BETAS, eps=1e-8, decay=0.1, max_norm=None, std=0.1, seed=5, first=False, **kw):
    g = _gen(len(sizes) * 1000 + sum(sizes) % 997 + bits)
    ps, gs = [_normal(g, n, dtype=p_type) for n in sizes], [_normal(g, n, dtype=g_type, std=std) for n in sizes]
    ss = [tuple(torch.zeros_like(t) for t in _state(g, n, bits, std)) if first else _state(g, n, bits, std) for n in sizes]
    offsets = [(3 * k) % 5 for k in range(len(sizes))]
    dev = [[_odd(t, o) for t, o in zip(ts, offsets)] for ts in (ps, gs, *zip(*ss))]
    copies = [_odd(torch.zeros(n, dtype=copy), o) for n, o in zip(sizes, offsets)] if copy else None
    norm = None if max_norm is None else torch.stack([t.double().square().sum() for t in gs]).sum().sqrt().float()
    views = [[v for v, _ in d] for d in dev]
    decays = [float(torch.tensor(d)) for d in (decay if isinstance(decay, list) else [decay] * len(sizes))]
    features.adamw(views[0], views[1], list(zip(*views[2:])), step, lr=lr, betas=betas, eps=eps, weight_decay=decay, norm=None if norm is None else norm.to(DEV),
                   max_norm=1.0 if max_norm is None else max_norm, copies=None if copies is None else [v for v, _ in copies], seed=seed, **kw)
    # every step of the state of the tensors is between 0 and 4, so that they begin at odd places
    for k, n in enumerate(sizes):
        for d in dev:
            blocks = d[k][0].numel()
            assert _around(d[k][1], offsets[k], blocks), k
        assert torch.equal(views[1][k].cpu(), gs[k])
        want = to.adamw(ps[k], gs[k], ss[k], step, lr, betas, float(torch.tensor(eps)), decays[k], None if norm is None else float(norm),
                        1.0 if max_norm is None else float(torch.tensor(max_norm)), copy, seed, place=k)
        fo.close(views[0][k], want["param"], f"param {k}")
        if copy:
            fo.close(copies[k][0], want["copy"], f"copy {k}")
            assert _around(copies[k][1], offsets[k], n)
        if bits == 32:
            fo.close(views[2][k], want["m"], f"m {k}")
            fo.close(views[3][k], want["v"], f"v {k}")
        else:
            fo.close(views[4][k], want["m_scale"], f"m_scale {k}")
            fo.close(views[5][k], want["r_scale"], f"r_scale {k}")
            to.between(views[2][k], want["m"], f"m {k}")
            to.between(views[3][k], want["r"], f"r {k}")
    return views


# One element, both sides of a vector, of a block and of a chunk, and none.
SIZES = [1, 3, 4, 5, 0, 255, 256, 257, 1023, 1024, 1025, 4097, 10_000, 2, 777]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p,g", TYPES)
def test_adamw_types(p, g, bits):
    _check_step(SIZES, p, g, bits)
    _check_step(SIZES, p, g, bits, max_norm=1.0, std=3.0)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("copy", [BF16, F16])
def test_adamw_copies(copy, bits):
    _check_step(SIZES, F32, BF16, bits, copy=copy)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kw", [dict(step=1, first=True), dict(step=2, betas=(0.0, 0.0)), dict(step=100_000), dict(lr=0.0), dict(decay=0.0), dict(eps=1e-3), dict(lr=1.0, decay=0.9),
                                dict(max_norm=1e6), dict(max_norm=0.0), dict(std=1e-6), dict(std=1e4), dict(decay=[0.1 * k for k in range(15)]), dict(seed=0xFFFFFFFF),
                                dict(betas=(0.5, 0.9999)), dict(step=1 << 40)])
def test_adamw_settings(kw, bits):
    _check_step(SIZES, F32, F32, bits, **kw)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_many_tensors_and_whole_chunks(bits):
    _check_step([1 + (i * 37) % 611 for i in range(150)], F32, BF16, bits, copy=BF16)  # several launches
    _check_step([1_200_001, 5, 300_000], BF16, BF16, bits)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_large_chunks(bits):
    # Enough elements for the large chunks and for workgroups of several, on the GPU in 64 bits.
    g = torch.Generator(device=DEV).manual_seed(bits)
    n = [9_000_001, 77, 600_000]
    ps, gs = [torch.randn(k, device=DEV, generator=g) for k in n], [torch.randn(k, device=DEV, generator=g) * 0.1 for k in n]
    before = [p.clone() for p in ps]
    state = features.adamw_state(ps, bits)
    features.adamw(ps, gs, state, 1, lr=1e-3, weight_decay=0.0)
    for p, b, grad, s in zip(ps, before, gs, state):
        # after the first step every parameter has moved by lr towards its gradient's sign
        moved = (b.double() - p.double()) / 1e-3
        assert ((moved - torch.sign(grad.double())).abs() <= 2e-4 * (1 + b.abs().double()) + 1e-8 / grad.abs().double()).all()
        if bits == 32:
            assert ((s[0].double() - 0.1 * grad.double()).abs() <= 3 * fo.U * 0.1 * grad.abs().double()).all()
        else:
            per = s[2].repeat_interleave(to.BLOCK)[:p.numel()].double()
            m = s[0].float().double() * per
            off = (m - 0.1 * grad.double()).abs()
            assert (off <= to.grid(0.1 * grad.double() / per) * per * (1 + 1e-5)).all()
            # rounded up and down alike
            assert abs(float((m - 0.1 * grad.double()).sum() / off.square().sum().sqrt())) < 6


# Enough elements to go past the caches, of every type, at the lines' beginnings and at odd places; a million are compared.
@pytest.mark.parametrize("offset", [0, 3])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p,g", TYPES)
def test_adamw_past_the_caches(p, g, bits, offset):
    gen = torch.Generator(device=DEV).manual_seed(bits)
    n, most = [13_500_001, 70_001], 1_000_192
    ps, gs = [torch.randn(k, device=DEV, generator=gen).to(p) for k in n], [(torch.randn(k, device=DEV, generator=gen) * 0.1).to(g) for k in n]
    state = features.adamw_state(ps, bits)
    copy = BF16 if p == F32 else None
    copies = [torch.zeros(k, dtype=BF16, device=DEV) for k in n] if copy else None
    if offset:
        wholes = []

        def moved(t):
            whole = torch.ones(t.numel() + 16, device=DEV).to(t.dtype)
            whole[offset:offset + t.numel()].copy_(t)
            wholes.append((whole, t.numel()))
            return whole[offset:offset + t.numel()]

        ps, gs, state = [moved(t) for t in ps], [moved(t) for t in gs], [tuple(moved(t) for t in st) for st in state]
        copies = [moved(t) for t in copies] if copy else None
    norm = features.grad_norm(gs)
    for t in (1, 2):
        before = [(q.clone(), tuple(s.clone() for s in st)) for q, st in zip(ps, state)]
        features.adamw(ps, gs, state, t, lr=1e-2, norm=norm, max_norm=3.0, copies=copies, seed=9)
        for k, (q, st) in enumerate(before):
            m = min(most, n[k])
            part = tuple(s[:m] if s.numel() == n[k] else s[:-(-m // to.BLOCK)] for s in st)
            want = to.adamw(q[:m], gs[k][:m], part, t, 1e-2, BETAS, float(torch.tensor(1e-8)), float(torch.tensor(0.01)), float(norm), 3.0, copy, 9, place=k)
            want = {name: tuple(w.cpu() for w in v) for name, v in want.items()}
            fo.close(ps[k][:m], want["param"], "param")
            if copy:
                fo.close(copies[k][:m], want["copy"], "copy")
            if bits == 32:
                fo.close(state[k][0][:m], want["m"], "m")
                fo.close(state[k][1][:m], want["v"], "v")
            else:
                to.between(state[k][0][:m], want["m"], "m")
                to.between(state[k][1][:m], want["r"], "r")
                fo.close(state[k][2][:-(-m // to.BLOCK)], want["m_scale"], "m_scale")
                fo.close(state[k][3][:-(-m // to.BLOCK)], want["r_scale"], "r_scale")
            last = slice(n[k] - 5, n[k])
            assert (ps[k][last] != q[last]).any()
    if offset:
        assert all((w[:offset].float() == 1).all() and (w[offset + m:].float() == 1).all() for w, m in wholes)


def test_adamw_takes_scalars_from_the_gpu():
    g = _gen(9)
    for bits in (32, 8):
        outs = []
        for on_gpu in (False, True):
            gg = _gen(77)
            p, grad = _normal(gg, 3000).to(DEV), _normal(gg, 3000).to(DEV)
            state = [tuple(t.to(DEV) for t in _state(gg, 3000, bits, 1.0))]
            for t in (5, 6):
                step, lr = (torch.tensor(t, device=DEV), torch.tensor(0.0078125, device=DEV)) if on_gpu else (t, 0.0078125)
                features.adamw([p], [grad], state, step, lr=lr)
            outs.append([p] + [t.float() for t in state[0]])
        assert all(torch.equal(a, b) for a, b in zip(*outs))
    p = torch.ones(4, device=DEV)
    state = features.adamw_state([p])
    features.adamw([p], [p.clone()], state, torch.tensor([0], device=DEV), lr=0.5, weight_decay=0.0)  # counts as the first step
    assert torch.allclose(p, torch.full_like(p, 0.5))


def test_adamw_extremes():
    for bits in (32, 8):
        p = torch.ones(1000, device=DEV)
        grad = torch.ones(1000, device=DEV)
        grad[3], grad[500] = float("nan"), float("inf")
        state = features.adamw_state([p], bits)
        features.adamw([p], [grad], state, 1, lr=0.1, weight_decay=0.0)
        there = torch.isnan(p).nonzero().view(-1).tolist()
        assert there == [3, 500]
        rest = [k for k in range(1000) if k not in there]
        assert torch.allclose(p[rest], torch.full((998,), 0.9, device=DEV))
        if bits == 8:  # the others of their blocks keep their states and scales
            m, r, ms, rs = state[0]
            assert torch.isnan(m.float()).nonzero().view(-1).tolist() == there and torch.isnan(r.float()).nonzero().view(-1).tolist() == there
            assert (m.float()[rest] == to.TOP).all() and (r.float()[rest] == to.TOP).all()
            assert torch.allclose(ms, torch.full_like(ms, 0.1 / to.TOP)) and torch.allclose(rs, torch.full_like(rs, 0.001 ** 0.5 / to.TOP))
        # a zero gradient and state leave the parameters to the decay, and no NaN
        p = torch.full((300,), 2.0, device=DEV)
        state = features.adamw_state([p], bits)
        features.adamw([p], [torch.zeros_like(p)], state, 1, lr=0.5, weight_decay=0.5)
        assert (p == 1.5).all() and not any(t.float()[:2].any() for t in state[0][:2])
        # an infinite norm takes the gradients away, a NaN spoils them
        for value in (float("inf"), float("nan")):
            p, grad = torch.ones(20, device=DEV), torch.ones(20, device=DEV)
            state = features.adamw_state([p], bits)
            features.adamw([p], [grad], state, 1, lr=0.5, weight_decay=0.0, norm=torch.tensor(value, device=DEV))
            assert torch.isnan(p).all() if value != value else (p == 1).all()


def test_states_of_8_bits_follow_small_changes():
    # Gradients of one size for hundreds of steps: the second moment rises to it, though a step changes it by a thousandth.
    torch.manual_seed(0)
    n, size = 4096, torch.logspace(-2, 0, 4096, device=DEV)
    p = torch.zeros(n, device=DEV)
    state = features.adamw_state([p], 8)
    b2 = 0.99
    for t in range(1, 801):
        features.adamw([p], [size * (1 - 2 * (torch.rand(n, device=DEV) < 0.5).float())], state, t, lr=0.0, betas=(0.9, b2), weight_decay=0.0)
    m, r, ms, rs = state[0]
    v = (r.float() * rs.repeat_interleave(to.BLOCK)).square() / size.square()
    # E v = (1 - b2^800) size^2 = 0.9997 size^2.  In a step v moves by up to 1 % of itself, its variance by at most step^2 times that
    # share of a step of r^2 (1/4 of itself): 0.0025 v^2 at most, over 1 / (1 - b2^2) = 50 steps 0.13 v^2; the mean over 4,096
    # elements has a standard deviation of at most 0.36 / 64 = 0.006, of which six are 0.034.
    assert abs(float(v.double().mean()) - 0.9997) < 0.034
    assert not (r.float() == 0).any()


# ---------------------------------------------------------------- whole steps, streams, graphs


def _make(seed, bits, n=6000, rows=700, dim=48, copies=False):
    g = _gen(seed)
    t = {"ids": torch.randint(-1, rows, (n,), generator=g).to(DEV), "table": _normal(g, rows, dim).to(DEV), "weight": (1 + _normal(g, dim, std=0.1)).to(DEV),
         "stream": _normal(g, n, dim).to(DEV), "dy": _normal(g, n, dim).to(DEV), "more": _normal(g, n, dim, std=0.1).to(DEV),
         "step": torch.tensor(0, device=DEV), "lr": torch.tensor(0.01, device=DEV)}
    t["state"] = features.adamw_state([t["table"], t["weight"]], bits)
    t["copies"] = [torch.zeros(rows, dim, dtype=BF16, device=DEV), None] if copies else None
    return t


def _train(t, stream=None):
    x = features.embed(t["ids"], t["table"], scale=4.0, stream=stream)
    y, rstd, h = features.rms_norm(x, t["weight"], t["stream"], stream=stream)
    q, scale, _, _ = features.rms_norm_8bit(x, t["weight"], t["stream"], group=32, stream=stream)
    dh, dw = features.rms_norm_grad(t["dy"], h, rstd, t["weight"], t["more"], stream=stream)
    dtable = features.embed_grad(t["ids"], dh, t["table"].shape[0], scale=4.0, stream=stream)
    norm = features.grad_norm([dtable, dw], stream=stream)
    with torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.current_stream() if stream is None else torch.cuda.ExternalStream(stream)):
        t["step"].add_(1)
    features.adamw([t["table"], t["weight"]], [dtable, dw], t["state"], t["step"], lr=t["lr"], weight_decay=[0.1, 0.0], norm=norm, max_norm=0.5,
                   copies=t["copies"], seed=11, stream=stream)
    return y, q.float(), scale, dtable, dw, norm


def _held(t):
    return [t["table"], t["weight"]] + [s.float() for state in t["state"] for s in state] + ([t["copies"][0]] if t["copies"] else [])


@pytest.mark.parametrize("bits", [32, 8])
def test_training_step_is_what_its_parts_are(bits):
    t = _make(1, bits, copies=True)
    before = {k: t[k].clone() for k in ("table", "weight")}
    y, q, scale, dtable, dw, norm = _train(t)
    x, w = features.embed(t["ids"], before["table"], scale=4.0).cpu(), before["weight"].cpu()
    h = to.stream(x, t["stream"].cpu())
    want, (rstd, _) = to.rms_norm(h, w, float(torch.tensor(1e-6)))
    fo.close(y, want, "y")
    for k, (name, grad) in enumerate((("table", dtable), ("weight", dw))):
        zeros = tuple(torch.zeros_like(s).cpu() for s in t["state"][k])
        out = to.adamw(before[name].cpu(), grad.cpu(), zeros, 1, float(torch.tensor(0.01)), BETAS, float(torch.tensor(1e-8)), [float(torch.tensor(0.1)), 0.0][k],
                       float(norm), 0.5, BF16 if k == 0 else None, 11, place=k)
        fo.close(t[name], out["param"], name)
        if k == 0:
            fo.close(t["copies"][0], out["copy"], "copy")


@pytest.mark.parametrize("bits", [32, 8])
def test_training_on_another_stream(bits):
    a, b, c = (_make(2, bits, copies=True) for _ in range(3))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        want = _train(a)
        for other, stream in ((b, side), (c, side.cuda_stream)):
            got = _train(other, stream)
            side.synchronize()
            torch.cuda.synchronize()
            assert all(torch.equal(u, v) for u, v in zip(got, want))
    for other in (b, c):
        assert all(torch.equal(u, v) for u, v in zip(_held(a), _held(other)))


@pytest.mark.parametrize("bits", [32, 8])
def test_training_in_a_graph(bits):
    eager, static, other = _make(3, bits), _make(3, bits), _make(4, bits)
    _train(_make(5, bits))  # loads the kernels
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _train(static)
    for k in range(5):
        for t in (eager, static):
            t["lr"].fill_(0.01 / (k + 1))
            if k == 2:
                t["dy"].copy_(other["dy"])
                t["ids"].copy_(other["ids"])
        graph.replay()
        want = _train(eager)
        torch.cuda.synchronize()
        assert int(static["step"]) == int(eager["step"]) == k + 1
        assert all(torch.equal(u, v) for u, v in zip(outs, want))
        assert all(torch.equal(u, v) for u, v in zip(_held(eager), _held(static)))


def test_two_graphs_with_gradients_share_nothing():
    a, b = _make(6, 8), _make(7, 8)
    ea, eb = _make(6, 8), _make(7, 8)
    _train(_make(5, 8))
    torch.cuda.synchronize()
    ga, gb = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(ga):
        oa = _train(a)
    with torch.cuda.graph(gb):
        ob = _train(b)
    side = torch.cuda.Stream()
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        ga.replay()
        with torch.cuda.stream(side):
            gb.replay()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        for outs, e in ((oa, ea), (ob, eb)):
            want = _train(e)
            torch.cuda.synchronize()
            assert all(torch.equal(u, v) for u, v in zip(outs, want))
    assert all(torch.equal(u, v) for u, v in zip(_held(a) + _held(b), _held(ea) + _held(eb)))


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_clips_as_clip_grads_does(bits):
    # A step by gradients clipped before and one that clips on the way: the same within the roundings of the clipped ones.
    g = _gen(10)
    p0, grad = _normal(g, 5000), _normal(g, 5000)
    out = []
    for fused in (True, False):
        p, d = p0.to(DEV), grad.to(DEV)
        state = features.adamw_state([p], bits)
        if fused:
            features.adamw([p], [d], state, 1, lr=0.1, norm=features.grad_norm([d]), max_norm=0.5)
        else:
            features.clip_grads([d], 0.5)
            features.adamw([p], [d], state, 1, lr=0.1)
        out.append(p.double())
    # lr m / (sqrt(v) + eps) is lr in size and off by some u of itself, the parameters by theirs
    assert ((out[0] - out[1]).abs() <= 0.1 * 16 * fo.U + 4 * fo.U * out[0].abs()).all()


# ---------------------------------------------------------------- refusals and autograd


def test_adamw_refusals():
    def call(p=None, g=None, s=None, step=1, **kw):
        p = [torch.ones(300, device=DEV)] if p is None else p
        g = [torch.ones(300, device=DEV)] if g is None else g
        s = features.adamw_state(p) if s is None else s
        return lambda: features.adamw(p, g, s, step, **kw)

    one = torch.ones(300, device=DEV)
    eight = features.adamw_state([one], 8)[0]
    whole = torch.ones(1000, device=DEV)
    half = one.half()
    bad = [
        call(p=[], g=[], s=[]), call(g=[]), call(s=[]), call(p=[one.cpu()], s=features.adamw_state([one])), call(g=[one.cpu()]), call(g=[one[:299]]), call(g=[one.view(3, 100)]),
        call(p=[one.double()]), call(g=[one.double()]), call(p=[torch.ones(300, 2, device=DEV)[:, 0]], s=features.adamw_state([one])), call(g=[torch.ones(300, 2, device=DEV)[:, 0]]),
        call(s=[(one,)]), call(s=[(one, one.clone(), one.clone())]), call(s=[(one, half)]), call(s=[(one.clone(), one[:299].clone())]), call(s=[(one.clone(), one.cpu())]),
        call(s=[iter((one.clone(), one.clone()))]),
        call(s=[(eight[0], eight[1], eight[2][:1], eight[3])]), call(s=[(eight[0], eight[1], eight[2], eight[3].double())]), call(s=[(eight[0], one.clone(), eight[2], eight[3])]),
        call(s=[(eight[0], eight[1])]), call(copies=[one.clone()]), call(copies=[]), call(copies=[half[:299]]), call(p=[half], g=[half.clone()], copies=[half.clone()]),
        call(weight_decay=[0.1, 0.2]), call(seed=-1), call(seed=1 << 32), call(step=torch.tensor(1)), call(step=torch.tensor(1.0, device=DEV)),
        call(step=torch.ones(2, dtype=torch.int64, device=DEV)), call(lr=torch.tensor(0.1)), call(lr=torch.tensor(0.1, device=DEV, dtype=torch.float64)),
        call(norm=torch.ones(2, device=DEV)), call(norm=torch.tensor(1.0)),
        # shared memory
        call(p=[one, one], g=[one.clone(), one.clone()], s=features.adamw_state([one, one])), call(p=[one], g=[one]), call(p=[whole[:300]], g=[whole[299:599]]),
        call(s=[(one, one)]), call(p=[one], s=[(one, one.clone())]), call(p=[whole[:300]], norm=whole[5:6]), call(p=[whole[:300]], lr=whole[5]),
        call(p=[whole[:300], whole[200:500]], g=[one, one], s=features.adamw_state([one, one])),
        call(s=[(eight[0], eight[0], eight[2], eight[3])]), call(s=[(eight[0], eight[1], eight[2], eight[2])]),
    ]
    for k, f in enumerate(bad):
        with pytest.raises(ValueError):
            print("refusal", k)
            f()
    for f in (call(lr=-1.0), call(step=0), call(betas=(1.0, 0.9)), call(betas=(0.9, -0.1)), call(eps=-1.0), call(weight_decay=-1.0), call(norm=torch.tensor(1.0, device=DEV), max_norm=-1.0),
              call(p=[half], g=[half.bfloat16()], s=features.adamw_state([half]))):
        with pytest.raises(scd.ScdError):
            f()
    for f in (lambda: features.adamw_state([one], 16), lambda: features.adamw_state([one], 4)):
        with pytest.raises(ValueError):
            f()


def test_adamw_and_autograd():
    p = torch.nn.Parameter(torch.ones(300, device=DEV))
    grad, state = torch.ones(300, device=DEV), features.adamw_state([p])
    with pytest.raises(ValueError, match="requires gradients"):
        features.adamw([p], [grad], state, 1)
    assert not any(t.any() for t in state[0]) and (p == 1).all()
    saved = (p * p).sum()  # keeps p for its backward pass
    versions = [t._version for t in (p, grad, *state[0])]
    with torch.no_grad():
        features.adamw([p], (grad,), iter(state), 1, lr=0.5, weight_decay=iter([0.0]))
    assert [t._version - v for t, v in zip((p, grad, *state[0]), versions)] == [1, 0, 1, 1]
    assert torch.allclose(p.detach(), torch.full_like(p, 0.5))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        saved.backward()


def test_example_runs_with_the_step():
    import math
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import learned_features
    objectives = learned_features.train(iterations=3, n=2048, adamw=True)
    assert len(objectives) == 3 and all(math.isfinite(p) for p in objectives)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_offsets_beyond_32_bits(bits):
    n = (1 << 32) + 1000
    at = [0, 5, 255, (1 << 31) + 7, (1 << 32) - 1, 1 << 32, (1 << 32) + 5, n - 1]
    p, grad = (torch.zeros(n, dtype=BF16, device=DEV) for _ in range(2))
    state = features.adamw_state([p], bits)
    values = torch.arange(1.0, len(at) + 1).bfloat16()
    grad[torch.tensor(at, device=DEV)] = values.to(DEV)
    features.adamw([p], [grad], state, 1, lr=0.25, weight_decay=0.0, seed=3)
    assert int((p != 0).sum()) == len(at)
    assert (p[torch.tensor(at, device=DEV)] == -0.25).all()
    if bits == 32:
        m = state[0][0][torch.tensor(at, device=DEV)].cpu()
        assert ((m.double() - 0.1 * values.double()).abs() <= 3 * fo.U * 0.1 * values.double()).all()
        return
    for first in (0, (1 << 32) - 256, 1 << 32):  # whole blocks, whose words come from beyond 32 bits
        here = slice(first, first + 256)
        g = grad[here].double().cpu()
        block = first // 256
        for q, s, value, which, to_8 in ((state[0][0], state[0][2], 0.1 * g, 0, to.round_m), (state[0][1], state[0][3], (0.001 * g * g).sqrt(), 1, to.round_r)):
            scale = s[block].double().cpu()
            assert abs(float(scale) * to.TOP / float(value.max()) - 1) < 1e-6
            u = to.uniform(to.words(256, 3, 1, 0, start=first))[which]
            least, most = to_8(value / scale * (1 - 1e-6), u), to_8(value / scale * (1 + 1e-6), u)
            to.between(q[here], (least, most, torch.sign(value)), f"{first} {which}")
