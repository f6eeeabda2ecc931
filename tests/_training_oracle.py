"""Plain 64-bit implementations of the root-mean-square norm, its gradient and the AdamW step, on the CPU, with the bounds
that a 32-bit computation of them keeps (as in _features_oracle.py: u = 2^-24, first-order terms, SLACK for the rest).

Values of 8 bits are e4m3: neighbours lie 2^(e - 3) apart in [2^e, 2^(e + 1)), 2^-9 below 2^-6.
"""
import math

import torch

import _features_oracle as fo
from _features_oracle import SLACK, U

TOP = 448.0
TINY = 2.0 ** -126
BLOCK = 256
E4M3 = torch.float8_e4m3fn


def rounded(value, error, dtype):
    return SLACK * error if dtype == torch.float64 else fo.rounded(value, error, dtype)


def depth(dim):
    """Additions on the way of a term through a row's sum: at most 64 elements in a lane, or a vector more than the row's
    1024th part, 6 steps of the wave's tree and up to 16 waves."""
    return max(64, dim // 1024 + 8) + 6 + 16


def grid(x):
    """The distance of neighbouring values of 8 bits around |x|."""
    e = x.abs().clamp(min=2.0 ** -6).double().view(torch.int64) >> 52  # the exponent's bits: exact on every device
    return ((e - 3) << 52).view(torch.float64).to(x.dtype)


def stream(x, residual):
    """What is normalised: the sum in 32 bits, rounded to the type."""
    return x if residual is None else (x.float() + residual.float()).to(x.dtype)


def _rms(h, weight, eps):
    h = h.double()
    dim = h.shape[-1]
    w = torch.ones(dim, dtype=torch.float64) if weight is None else weight.double()
    ms = h.square().mean(-1, keepdim=True)
    rstd = (ms + eps).rsqrt()
    # squares and their sum, the division by dim and the addition of eps; then the root and the inverse
    e_rstd = rstd * (0.5 * (depth(dim) + 4) * U * ms * rstd.square() + 4 * U)
    y = h * rstd * w
    return y, y.abs() * (e_rstd / rstd + 3 * U), rstd, e_rstd


def rms_norm(h, weight, eps):
    y, e_y, rstd, e_rstd = _rms(h, weight, eps)
    return (y, rounded(y, e_y, h.dtype)), (rstd[..., 0], SLACK * e_rstd[..., 0])


def rms_norm_8bit(h, weight, eps, group):
    """((q, bound), (scale, bound)): q before its rounding, with half a step more."""
    y, e_y, _, _ = _rms(h, weight, eps)
    rows, dim = y.shape
    g = group or dim

    def tops(t):
        return torch.nn.functional.pad(t, (0, -dim % g)).view(rows, -1, g).abs().amax(2)

    top = tops(y) / TOP
    scale = top.clamp(min=TINY)
    e_scale = tops(e_y) / TOP + 2 * U * scale
    per = scale.repeat_interleave(g, 1)[:, :dim]
    z = y / per
    e_z = (e_y + z.abs() * e_scale.repeat_interleave(g, 1)[:, :dim]) / per + 3 * U * z.abs()
    half = grid(z) / 2  # z beyond a power of two by its error lies within half a step of that value all the same
    if not group:
        scale, e_scale = scale[:, 0], e_scale[:, 0]
    return (z, SLACK * e_z + half), (scale, SLACK * e_scale)


def rms_norm_grad(dy, h, rstd, weight, residual, dtype, param_dtype):
    dim = h.shape[-1]
    dy, h, rstd = dy.double().reshape(-1, dim), h.double().reshape(-1, dim), rstd.double().reshape(-1, 1)
    w = torch.ones(dim, dtype=torch.float64) if weight is None else weight.double()
    n = h * rstd
    g = dy * w
    c = (g * n).mean(-1, keepdim=True)
    dx = rstd * (g - n * c)
    d = depth(dim)
    e_c = (d + 5) * U * (g * n).abs().mean(-1, keepdim=True)
    e_dx = rstd.abs() * (n.abs() * e_c + 5 * U * (g.abs() + (n * c).abs()))
    if residual is not None:
        dx = dx + residual.double().reshape(-1, dim)
        e_dx = e_dx + U * dx.abs()
    dw = (dy * n).sum(0)
    return (dx, rounded(dx, e_dx, dtype)), (dw, rounded(dw, (h.shape[0] + 3) * U * (dy * n).abs().sum(0), param_dtype))


# ---------------------------------------------------------------- AdamW


def mix(h):
    """The finaliser of MurmurHash3, of a number or a tensor of them below 2^32."""
    h = ((h ^ (h >> 16)) * 0x85EBCA6B) & 0xFFFFFFFF
    h = ((h ^ (h >> 13)) * 0xC2B2AE35) & 0xFFFFFFFF
    return h ^ (h >> 16)


def words(n, seed, step, place, start=0, device="cpu"):
    key = mix((mix(seed ^ mix(step & 0xFFFFFFFF)) + place) & 0xFFFFFFFF)
    at = torch.arange(start, start + n, dtype=torch.int64, device=device)
    return mix((at & 0xFFFFFFFF) ^ ((key + (at >> 32)) & 0xFFFFFFFF))


def uniform(word):
    """The numbers that m and sqrt(v) are rounded with."""
    return ((word & 0xFFFF).double() + 0.5) / 65536, ((word >> 16).double() + 0.5) / 65536


def round_m(z, u):
    """|z| >= 0 goes up with the probability that keeps its mean."""
    step = grid(z)
    low = torch.floor(z / step) * step
    return torch.where(z - low > u * step, low + step, low).clamp(max=TOP)


def round_r(z, u):
    """z >= 0 goes up with the probability that keeps the mean of its square, and always from between 0 and the least value."""
    step = grid(z)
    low = torch.floor(z / step) * step
    up = z.square() - low.square() > u * ((low + step).square() - low.square())
    return torch.where(up | ((low == 0) & (z > 0)), low + step, low).clamp(max=TOP)


def blocks(x, fill=0.0):
    return torch.nn.functional.pad(x.reshape(-1), (0, -x.numel() % BLOCK), value=fill).view(-1, BLOCK)


def decode(state):
    """(m, v) in 64 bits of a state of either kind."""
    if len(state) == 2:
        return state[0].double(), state[1].double()
    n, shape = state[0].numel(), state[0].shape
    m, r = (blocks(q.float().double()) * s.double()[:, None] for q, s in ((state[0], state[2]), (state[1], state[3])))
    return m.view(-1)[:n].view(shape), (r * r).view(-1)[:n].view(shape)


def adamw(p, grad, state, step, lr, betas, eps, decay, norm=None, max_norm=1.0, copy=None, seed=0, place=0):
    """The new values, each with its bound: {"param", "m", "v" (32 bits)} or {"param", "m", "r", "m_scale", "r_scale"}, where
    m and r are (least, most) values in 8 bits; and "copy"."""
    b1, b2 = betas
    m0, v0 = decode(state)
    if norm is not None and not norm <= max_norm:
        factor = max_norm / norm
    else:
        factor = 1.0
    g = grad.double() * factor
    eight = len(state) == 4
    m = b1 * m0 + (1 - b1) * g
    v = b2 * v0 + (1 - b2) * g * g
    # the betas as 32-bit numbers, two roundings of g, the products and the sum; one more for a state that is decoded
    e_m = 5 * U * (b1 * m0.abs() + (1 - b1) * g.abs())
    e_v = 9 * U * v
    root = (v / (1 - b2 ** step)).sqrt() + eps
    move = lr / (1 - b1 ** step) * m / root
    move = torch.where(m == 0, torch.where(root == 0, math.nan, 0.0), move)
    # sqrt halves the variance's error; the two factors, root, product, sum and quotient round once each
    e_move = lr / (1 - b1 ** step) * e_m / root + 12 * U * move.abs()
    kept = p.double() * (1 - lr * decay)
    new = kept - move
    e_p = torch.nan_to_num(e_move) + 2 * U * kept.abs() + U * new.abs()
    out = {"param": (new, rounded(new, e_p, p.dtype))}
    if copy is not None:
        out["copy"] = (new, rounded(new, e_p, copy))
    if not eight:
        out["m"], out["v"] = (m, SLACK * e_m + 2.0 ** -149), (v, SLACK * e_v + 2.0 ** -148)
        return out
    um, ur = uniform(words(p.numel(), seed, step, place, device=p.device))
    r = v.sqrt()
    e_r = (0.5 * 9 + 1) * U * r
    for name, x, e, u, to in (("m", m, e_m, um, round_m), ("r", r, e_r, ur, round_r)):
        top = blocks(x.abs()).amax(1)
        scale = (top / TOP).clamp(min=TINY)
        e_scale = SLACK * (blocks(e).amax(1) / TOP + 2 * U * scale)
        per = scale.repeat_interleave(BLOCK)[:x.numel()]
        z = x.reshape(-1).abs() / per
        e_z = SLACK * (e.reshape(-1) / per + z * (e_scale.repeat_interleave(BLOCK)[:x.numel()] / per + 3 * U))
        # what lies between two neighbours is compared in 20 bits: nothing is lost from 2^-6 on, where a value has as many below
        # its first four; below, bits under 2^-9 / 2^20 are
        e_z = e_z + torch.where(z < 2.0 ** -6, 2.0 ** -29, 0.0)
        least, most = to((z - e_z).clamp(min=0.0), u), to(z + e_z, u)
        out[name] = (least.view(p.shape), most.view(p.shape), torch.sign(x))
        out[name + "_scale"] = (scale, e_scale)
    return out


def between(got, want, what=""):
    """Asserts that values of 8 bits are those that the value's bound allows."""
    least, most, sign = (t.cpu() for t in want)
    got = got.detach().cpu().float().double()
    assert not torch.isnan(got).any(), f"{what}: NaN"
    bad = (got.abs() < least) | (got.abs() > most) | (got * sign < 0)
    if bad.any():
        i = int(bad.reshape(-1).nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values in 8 bits are wrong; at {i} got {float(got.reshape(-1)[i])}, "
                             f"want {float(least.reshape(-1)[i])} to {float(most.reshape(-1)[i])}, sign {float(sign.reshape(-1)[i])}")
