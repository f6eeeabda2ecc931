"""The AdamW step on the GPU at the limits of its arguments, against its 64-bit oracle (tests/_training_oracle.py)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import _features_oracle as fo  # noqa: E402
import _training_oracle as to  # noqa: E402
from paper_1702_07005_amd import features  # noqa: E402

DEV = "cuda"
BETAS = (0.9, 0.999)


# eps below the least normal number of 32 bits, at it, none, and so large that its inverse is below it.
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -149, 2.0 ** -140, 2.0 ** -127, 2.0 ** -126, 2.0 ** 100, 2.0 ** 101, 2.0 ** 127], ids=str)
def test_eps_of_every_size(eps, bits):
    g = torch.Generator().manual_seed(bits)
    n = 1000
    p, grad = torch.randn(n, generator=g), torch.randn(n, generator=g)
    if eps > 1.0:
        p *= 1e-30  # which lr m / eps moves
        grad *= 1e9
    if eps:
        grad[::3] = 0.0  # parameters that nothing moves: 0 / eps
    zeros = tuple(t.cpu() for t in features.adamw_state([p.to(DEV)], bits)[0])
    want = to.adamw(p, grad, zeros, 1, 0.125, BETAS, eps, 0.0)["param"]
    d, state = p.to(DEV), [tuple(t.to(DEV) for t in zeros)]
    features.adamw([d], [grad.to(DEV)], state, 1, lr=0.125, betas=BETAS, eps=eps, weight_decay=0.0)
    assert not torch.isnan(d).any()
    fo.close(d, want, "param")
    if eps:
        assert torch.equal(d[::3].cpu(), p[::3])


# ---------------------------------------------------------------- states of 8 bits, bit by bit

C448 = torch.tensor(1.0) / torch.tensor(448.0)


def _stated(values, u, power):
    """Codes (as the numbers they stand for) and scales of |m| (power 1) or sqrt(v) (2), blocks of 256, in the 32-bit operations
    that the C header states; torch divides on the CPU as IEEE 754 does."""
    n = values.numel()
    scale = (to.blocks(values).amax(1) * C448).clamp(min=to.TINY)
    z = values / scale.repeat_interleave(to.BLOCK)[:n]
    assert z.dtype == torch.float32
    if power == 1:
        z = torch.where(z < 2.0 ** -6, torch.floor(z * 2.0 ** 29) * 2.0 ** -29, z)
    else:
        z = torch.where(z > 0, z.clamp(min=2.0 ** -9), z)
    step = to.grid(z)
    low = torch.floor(z / step) * step
    u = u.float()
    up = z - low > u * step if power == 1 else (z - low) * (z + low) > step * u * (2 * low + step)
    return (low + up * step).clamp(max=to.TOP), scale


def _same_states(n, grads, start, step, betas, seed, **kw):
    params = [torch.zeros(k, device=DEV) for k in n]
    state = [tuple(t.to(DEV) for t in s) for s in start]
    features.adamw(params, [g.to(DEV) for g in grads], state, step, lr=0.0, betas=betas, seed=seed, **kw)
    b1, b2, a1, a2 = (torch.tensor(x, dtype=torch.float64).float() for x in (*betas, 1 - betas[0], 1 - betas[1]))
    for k, (g, s0, got) in enumerate(zip(grads, start, state)):
        m0, r0 = (q.float() * s.repeat_interleave(to.BLOCK)[:n[k]] for q, s in ((s0[0], s0[2]), (s0[1], s0[3])))
        g = g.float()
        m = b1 * m0 + a1 * g
        # torch's root of 32 bits is a unit off for some numbers on the CPU; one of 64 bits, whose rounding to 32 is the root's (no
        # root of a 24-bit number lies within 2^-26 of itself of the middle between two)
        r = (b2 * (r0 * r0) + a2 * (g * g)).double().sqrt().float()
        um, ur = to.uniform(to.words(n[k], seed, step, k))
        for name, q, scale, value, u, power in (("m", got[0], got[2], m.abs(), um, 1), ("r", got[1], got[3], r, ur, 2)):
            want, want_scale = _stated(value, u, power)
            if name == "m":
                want = want * torch.sign(m)
            assert torch.equal(scale.cpu(), want_scale), f"{name}_scale {k}"
            bad = q.float().cpu() != want
            assert not bad.any(), f"{name} {k}: {int(bad.sum())} of {n[k]} codes differ"
    return [tuple(t.cpu() for t in s) for s in state]


# Sizes of gradients down to where squares and scales leave the normal numbers, over steps that start from what the last one left.
@pytest.mark.parametrize("std", [1.0, 3e-3, 1e-12, 1e-19, 1e-22, 1e-30, 1e-37, 1e12])
@pytest.mark.parametrize("betas", [BETAS, (0.5, 0.9), (0.0, 0.0)])
def test_states_of_8_bits_are_those_of_the_stated_roundings(betas, std):
    g = torch.Generator().manual_seed(int(betas[0] * 10))
    n = [400_000, 1, 255, 257, 30_011]
    state = [tuple(t.cpu() for t in s) for s in features.adamw_state([torch.zeros(k, device=DEV) for k in n], 8)]
    for t in (1, 2, 9):
        grads = [torch.randn(k, generator=g) * torch.exp(2 * torch.randn(k, generator=g)) * std for k in n]
        state = _same_states(n, grads, state, t, betas, 77)


# ---------------------------------------------------------------- past the caches, every element


# Enough elements to go past the caches, at the lines' beginnings and at odd places: turns of 512 chunks on one XCD each, the
# chunks that fill none, and the last ones, all against the oracle.
@pytest.mark.parametrize("offset", [0, 3])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p,g", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16)], ids=str)
def test_every_element_past_the_caches(p, g, bits, offset, monkeypatch):
    gen = torch.Generator(device=DEV).manual_seed(bits + offset)
    n, part, seed, lr, step = [13_500_001, 70_001, 262_144 + 5], 1 << 20, 9, 1e-2, 3
    copy = torch.bfloat16 if p == torch.float32 else None

    def place(t):
        whole = torch.ones(t.numel() + 16, device=DEV).to(t.dtype)
        whole[offset:offset + t.numel()].copy_(t)
        return whole[offset:offset + t.numel()]

    ps = [place(torch.randn(k, device=DEV, generator=gen).to(p)) for k in n]
    gs = [place((torch.randn(k, device=DEV, generator=gen) * 0.1).to(g)) for k in n]
    state = [tuple(place(t) for t in s) for s in features.adamw_state(ps, bits)]
    copies = [place(torch.zeros(k, dtype=copy, device=DEV)) for k in n] if copy else None
    features.adamw(ps, gs, state, step - 1, lr=lr, seed=seed)
    before = [(q.clone(), tuple(s.clone() for s in st)) for q, st in zip(ps, state)]
    features.adamw(ps, gs, state, step, lr=lr, copies=copies, seed=seed)

    def within(got, want, what):
        value, bound = want
        bad = (got.double() - value).abs() > bound
        assert not (bad.any() or torch.isnan(got).any()), f"{what}: {int(bad.sum())} of {bad.numel()} outside"

    words = to.words
    for k, (q, st) in enumerate(before):
        for first in range(0, n[k], part):
            here = slice(first, min(first + part, n[k]))
            blocks = slice(first // to.BLOCK, -(-here.stop // to.BLOCK))
            monkeypatch.setattr(to, "words", lambda count, s, t, i, device: words(count, s, t, i, start=first, device=device))
            was = tuple(s[here] if s.numel() == n[k] else s[blocks] for s in st)
            now = tuple(s[here] if s.numel() == n[k] else s[blocks] for s in state[k])
            want = to.adamw(q[here], gs[k][here], was, step, lr, BETAS, float(torch.tensor(1e-8)), float(torch.tensor(0.01)), copy=copy, seed=seed, place=k)
            within(ps[k][here], want["param"], f"param {k} from {first}")
            if copy:
                within(copies[k][here], want["copy"], f"copy {k} from {first}")
            if bits == 32:
                within(now[0], want["m"], f"m {k} from {first}")
                within(now[1], want["v"], f"v {k} from {first}")
            else:
                within(now[2], want["m_scale"], f"m_scale {k} from {first}")
                within(now[3], want["r_scale"], f"r_scale {k} from {first}")
                to.between(now[0], want["m"], f"m {k} from {first}")
                to.between(now[1], want["r"], f"r {k} from {first}")


@pytest.fixture(scope="module", autouse=True)
def _give_back_memory():
    yield
    torch.cuda.empty_cache()
