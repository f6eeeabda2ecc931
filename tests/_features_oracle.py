"""Plain 64-bit implementations of the operators of learned features, on the CPU, with the bounds that a
32-bit computation of them keeps.

Each function returns the values and, for each, how far a correct kernel may be from it.  u = 2^-24 is the
rounding of 32-bit arithmetic; a sum of k terms formed in any order with at most d additions on the way of any
term is off by at most d u (sum of the terms' magnitudes) to first order; an output of p bits is rounded once
more, by at most 2^-p of its magnitude (or half the smallest subnormal).  Second-order terms are covered by
SLACK.
"""
import torch

U = 2.0 ** -24
SLACK = 1.05
ROUND = {torch.float32: (2.0 ** -24, 2.0 ** -150), torch.bfloat16: (2.0 ** -8, 2.0 ** -134), torch.float16: (2.0 ** -11, 2.0 ** -25)}


def rounded(value, error, dtype):
    """The bound of an output of `dtype` whose 32-bit value is off by at most `error`."""
    rel, least = ROUND[dtype]
    return SLACK * (error + rel * (value.abs() + error)) + least


def embed(tokens, table, scale, dtype):
    t = tokens.long()
    rows = table.shape[0]
    inside = (t >= 0) & (t < rows)
    full = torch.cat([table.double(), torch.zeros(1, table.shape[1], dtype=torch.float64)])
    v = full[torch.where(inside, t, rows)] * scale
    v[t < 0] = 0.0
    v[t >= rows] = float("nan")
    return v, rounded(v, U * v.abs(), dtype)


def embed_grad(tokens, grad, rows, scale, dtype, before=None):
    t = tokens.long().reshape(-1)
    g = grad.double().reshape(t.numel(), grad.shape[-1])
    inside = (t >= 0) & (t < rows)
    t, g = t[inside], g[inside]
    total = torch.zeros(rows, g.shape[1], dtype=torch.float64).index_add_(0, t, g)
    size = torch.zeros_like(total).index_add_(0, t, g.abs())
    count = torch.zeros(rows, dtype=torch.float64).index_add_(0, t, torch.ones(t.numel(), dtype=torch.float64))[:, None]
    v, e = total * scale, abs(scale) * (count + 1) * U * size
    if before is None:
        return v, torch.where(count > 0, rounded(v, e, dtype), 0.0)
    v = v + before.double()
    return v, torch.where(count > 0, rounded(v, e + U * v.abs(), dtype), 0.0)


def depth(dim):
    """Additions on the way of a term through a row's sum: at most 64 elements in a lane, 6 steps of the wave's tree
    and up to 16 waves; rows too wide for that have dim / 1024 elements in a lane."""
    return max(64, dim // 1024 + 1) + 6 + 16


def layer_norm(x, weight, bias, eps, dtype):
    x = x.double()
    dim = x.shape[-1]
    w = torch.ones(dim, dtype=torch.float64) if weight is None else weight.double()
    b = torch.zeros(dim, dtype=torch.float64) if bias is None else bias.double()
    mean = x.mean(-1, keepdim=True)
    c = x - mean
    var = c.square().mean(-1, keepdim=True)
    rstd = (var + eps).rsqrt()
    y = c * rstd * w + b
    d = depth(dim)
    e_mean = (d + 2) * U * x.abs().mean(-1, keepdim=True)
    e_c = e_mean + U * c.abs()
    # the centred values' common shift enters the variance squared, their roundings as they are
    e_var = e_mean.square() + (d + 4) * U * (var + e_mean.square()) + 2 * U * c.square().mean(-1, keepdim=True)
    e_rstd = rstd * (0.5 * e_var * rstd.square() + 4 * U)
    size = (c * rstd * w).abs()
    e_y = w.abs() * (rstd * e_c + c.abs() * e_rstd) + 3 * U * size + U * (size + b.abs())
    return (y, rounded(y, e_y, dtype)), (mean[..., 0], SLACK * e_mean[..., 0]), (rstd[..., 0], SLACK * e_rstd[..., 0])


def layer_norm_grad(dy, x, mean, rstd, weight, dtype, param_dtype):
    dim = x.shape[-1]
    dy, x = dy.double().reshape(-1, dim), x.double().reshape(-1, dim)
    mean, rstd = mean.double().reshape(-1, 1), rstd.double().reshape(-1, 1)
    w = torch.ones(dim, dtype=torch.float64) if weight is None else weight.double()
    h = (x - mean) * rstd  # off by 2 u of itself
    g = dy * w             # by u
    c1, c2 = g.mean(-1, keepdim=True), (g * h).mean(-1, keepdim=True)
    dx = rstd * (g - c1 - h * c2)
    dw, db = (dy * h).sum(0), dy.sum(0)
    d = depth(dim)
    e1 = (d + 3) * U * g.abs().mean(-1, keepdim=True)
    e2 = (d + 6) * U * (g * h).abs().mean(-1, keepdim=True)
    e_dx = rstd.abs() * (e1 + h.abs() * e2 + 6 * U * (g.abs() + c1.abs() + (h * c2).abs()))
    n = x.shape[0]
    return ((dx, rounded(dx, e_dx, dtype)), (dw, rounded(dw, (n + 4) * U * (dy * h).abs().sum(0), param_dtype)),
            (db, rounded(db, n * U * dy.abs().sum(0), param_dtype)))


def clip(grads, max_norm, dtypes):
    norm = torch.stack([g.double().square().sum() for g in grads]).sum().sqrt()
    factor = 1.0 if norm <= max_norm else max_norm / norm
    outs = []
    for g, t in zip(grads, dtypes):
        v = g.double() * factor
        outs.append((v, rounded(v, 2 * U * v.abs(), t)))
    return (norm, rounded(norm, 0.0 * norm, torch.float32)), outs


def close(got, want, what=""):
    """Asserts that `got` lies within its bound of the value, NaN where it is NaN."""
    value, bound = want
    got = got.detach().cpu().double().reshape(value.shape)
    nan = torch.isnan(value)
    assert torch.equal(torch.isnan(got), nan), f"{what}: NaN at other places"
    off = torch.where(nan, 0.0, (got - value).abs())
    bad = off > torch.where(nan, 0.0, bound)
    if bad.any():
        i = int(torch.where(bad, off - torch.where(nan, 0.0, bound), 0.0).reshape(-1).argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values outside their bound; at {i} got "
                             f"{float(got.reshape(-1)[i])!r}, want {float(value.reshape(-1)[i])!r} within {float(bound.reshape(-1)[i])!r}")
