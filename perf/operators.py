"""The operators of learned features, as cases whose time can be taken on one GPU.

A model of this library may read its coordinates from a table instead of from one-hot columns: ids are
looked up (``embed``), the vectors normalised (``layer_norm``), a linear read-out is fitted on them, and the
table is trained by the read-out's gradient, which goes back through both (``layer_norm_grad``,
``embed_grad``) and is clipped by its global norm (``clip``).

``listed`` holds the cases, ``draw`` gives further ones of the same ranges, ``prepare`` makes on the GPU what
a program holds before the call, ``run`` is the call (the operators' plain form where ``own`` is false, the
library's entry points where it is true), ``work`` counts what the call cannot do without, and ``exact``
computes the same outputs in 64 bits.

Ids follow Zipf's law inside each field (text has one field, click rows have 39), as in the library's own
text and click matrices, and a share of them is -1: padded places, which give zeros and receive nothing.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
FIELDS = 39  # of a click row


def listed():
    return [
        # One token of a model that answers token by token: what counts is the latency of the call.
        dict(name="embed_one_token", op="embed", tokens=1, rows=50_000, dim=4096, fields=1, table="bf16", out="bf16", wide_ids=True),
        # Click rows, 65,536 of them, every field an id into one table of narrow vectors.
        dict(name="embed_click_rows", op="embed", tokens=FIELDS * 65_536, rows=1_500_000, dim=16, fields=FIELDS, table="f32", out="f32", wide_ids=False),
        # A few sentences of a fine-tuning step, an odd width, gradients summed in a 32-bit table.
        dict(name="embed_grad_sentences", op="embed_grad", tokens=300, rows=4_999, dim=777, fields=1, grad="f16", table="f32", wide_ids=True),
        # A training step's text: frequent terms get hundreds of the rows, most of the table gets none.
        dict(name="embed_grad_text", op="embed_grad", tokens=16_384, rows=75_000, dim=1024, fields=1, grad="bf16", table="bf16", wide_ids=True),
        # The gradient of click rows: as many ids as table rows, vectors of 64 bytes.
        dict(name="embed_grad_click_rows", op="embed_grad", tokens=FIELDS * 32_768, rows=1_500_000, dim=16, fields=FIELDS, grad="f32", table="f32", wide_ids=False),
        # One token's features before they are scored.
        dict(name="norm_one_token", op="norm", rows=1, dim=4096, type="bf16", params="bf16", pad=0),
        # A training batch's features.
        dict(name="norm_batch", op="norm", rows=32_768, dim=2048, type="bf16", params="bf16", pad=0),
        # An odd number of rows that are part of a wider buffer, parameters kept in 32 bits.
        dict(name="norm_grad_view", op="norm_grad", rows=4_099, dim=1000, type="f16", params="f32", pad=24),
        # The concatenated vectors of click rows (39 x 16).
        dict(name="norm_grad_click_rows", op="norm_grad", rows=50_000, dim=FIELDS * 16, type="f32", params="f32", pad=0),
        # A training batch of wide features.
        dict(name="norm_grad_batch", op="norm_grad", rows=16_384, dim=4096, type="bf16", params="bf16", pad=0),
        # The gradients of a small read-out with its table and norms, at odd places of one buffer.
        dict(name="clip_small", op="clip", layers=2, width=61, rows=2_003, type="f32", out="f32", limit=1.0),
        # The gradients of a model of 350 M weights in half the width, clipped into what the update reads.
        dict(name="clip_model", op="clip", layers=12, width=2048, rows=50_000, type="bf16", out="f32", limit=1.0),
    ]


def _round(rng, lo, hi):
    """A size whose logarithm is spread evenly: half of them odd, half a power of two times 1, 5/4 or 7/4."""
    n = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    if rng.random() < 0.5:
        return min(int(n) | 1, hi)
    two = 2.0 ** math.floor(math.log2(n))
    return max(lo, min(hi, int(two * rng.choice((1, 1.25, 1.75)))))


def draw(rng):
    op = rng.choice(("embed", "embed_grad", "norm", "norm_grad", "clip"))
    kind = rng.choice(("f32", "bf16", "f16"))
    if op in ("embed", "embed_grad"):
        fields = rng.choice((1, 1, FIELDS))
        dim = _round(rng, 2, 256) if fields > 1 else _round(rng, 32, 8192)
        tokens = min(_round(rng, 1, 1 << 17) * fields, max(1, 80_000_000 // dim))
        rows = max(fields, min(_round(rng, 100, 2_000_000), 80_000_000 // dim))
        case = dict(op=op, tokens=tokens, rows=rows, dim=dim, fields=fields, wide_ids=rng.random() < 0.5)
        case["table"] = kind
        case["out" if op == "embed" else "grad"] = rng.choice((kind, kind, "bf16"))
        return case
    if op in ("norm", "norm_grad"):
        dim = _round(rng, 16, 16_384)
        rows = _round(rng, 1, max(1, min(1 << 18, 130_000_000 // dim)))
        return dict(op=op, rows=rows, dim=dim, type=kind, params=rng.choice((kind, "f32")), pad=rng.choice((0, 0, 8, 37)))
    width = _round(rng, 8, 2048)
    layers = _round(rng, 1, 64)
    rows = _round(rng, 1, 60_000)
    while layers * width * width * 5 + rows * width > 260_000_000:
        layers, rows = max(1, layers // 2), max(1, rows // 2)
    return dict(op=op, layers=layers, width=width, rows=rows, type=kind, out=rng.choice((kind, "f32")), limit=rng.choice((1.0, 1.0, 1e6)))


# --------------------------------------------------------------------------- inputs


def _zipf_ids(g, tokens, rows, fields):
    """Ids of Zipf(1) popularity inside each field's part of the table; popular ones lie apart; 2 % are -1."""
    place = torch.arange(tokens, device="cuda")
    part = rows // fields
    u = torch.rand(tokens, dtype=torch.float64, device="cuda", generator=g)
    rank = torch.expm1(u * math.log(part + 1)).floor().long().clamp_(0, part - 1)
    step = int(0.6180339887 * part) | 1
    while math.gcd(step, part) != 1:
        step += 2
    ids = (rank * step + 12_345) % part + place % fields * part
    none = torch.rand(tokens, device="cuda", generator=g) < 0.02
    return ids.masked_fill_(none & (place > 0), -1)


def _clip_shapes(case):
    w = case["width"]
    return [(case["rows"], w)] + [s for _ in range(case["layers"]) for s in ((w,), (w,), (w, w), (4 * w, w))]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, device="cuda", generator=g).mul_(std)

    state = {"case": case}
    op = case["op"]
    if op in ("embed", "embed_grad"):
        ids = _zipf_ids(g, case["tokens"], case["rows"], case["fields"])
        state["ids"] = ids if case["wide_ids"] else ids.int()
    if op == "embed":
        state["table"] = normal(case["rows"], case["dim"], std=0.02).to(TYPES[case["table"]])
        state["scale"] = math.sqrt(case["dim"])
    elif op == "embed_grad":
        state["grad"] = normal(case["tokens"], case["dim"], std=0.01).to(TYPES[case["grad"]])
        state["scale"] = math.sqrt(case["dim"])
    elif op in ("norm", "norm_grad"):
        rows, dim, kind = case["rows"], case["dim"], TYPES[case["type"]]
        # Features have a few channels that are larger than the others, and rows of their own sizes.
        channel = 1 + 7 * (torch.rand(dim, device="cuda", generator=g) < 0.01)
        size = torch.rand(rows, 1, device="cuda", generator=g) * 2 + 0.1
        x = torch.empty(rows, dim + case["pad"], dtype=kind, device="cuda")[:, :dim]
        x.copy_((normal(rows, dim) * channel + 0.3) * size)
        state["x"] = x
        state["weight"] = (1 + normal(dim, std=0.2)).to(TYPES[case["params"]])
        if op == "norm":
            state["bias"] = normal(dim, std=0.2).to(TYPES[case["params"]])
        else:
            state["grad"] = normal(rows, dim, std=0.01).to(kind)
            wide = x.double()
            mean = wide.mean(1)
            state["mean"] = mean.float()
            state["rstd"] = ((wide - mean[:, None]).square().mean(1) + EPS).rsqrt().float()
    else:
        shapes = _clip_shapes(case)
        sizes = [math.prod(s) for s in shapes]
        flat = normal(sum(sizes), std=0.003).to(TYPES[case["type"]])
        into = torch.empty_like(flat, dtype=TYPES[case["out"]])
        state["flat"], state["into"], state["limit"] = flat, into, case["limit"]
        state["grads"] = [t.view(s) for t, s in zip(flat.split(sizes), shapes)]
        state["outs"] = [t.view(s) for t, s in zip(into.split(sizes), shapes)]
    return state


# --------------------------------------------------------------------------- the call


def run(state):
    return _OWN[state["case"]["op"]](state) if own else _PLAIN[state["case"]["op"]](state)


def _plain_embed(s):
    ids = s["ids"].long()
    rows = s["table"][ids.clamp(min=0)].float() * s["scale"]
    return torch.where(ids[:, None] >= 0, rows, 0.0).to(TYPES[s["case"]["out"]])


def _plain_embed_grad(s):
    ids = s["ids"].long()
    rows = s["case"]["rows"]
    # the padded places' vectors go to a row after the last, which is left out
    total = torch.zeros(rows + 1, s["case"]["dim"], device="cuda")
    total.index_add_(0, torch.where(ids >= 0, ids, rows), s["grad"].float())
    return (total[:rows] * s["scale"]).to(TYPES[s["case"]["table"]])


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    x = x - mean
    rstd = (x.square().mean(1, keepdim=True) + EPS).rsqrt()
    y = x * rstd * s["weight"].float() + s["bias"].float()
    return {"y": y.to(s["x"].dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}


def _plain_norm_grad(s):
    grad, rstd = s["grad"].float(), s["rstd"][:, None]
    h = (s["x"].float() - s["mean"][:, None]) * rstd
    g = grad * s["weight"].float()
    dx = rstd * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    kind = s["weight"].dtype
    return {"x": dx.to(s["x"].dtype), "weight": (grad * h).sum(0).to(kind), "bias": grad.sum(0).to(kind)}


def _plain_clip(s):
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt()
    factor = torch.where(norm > s["limit"], s["limit"] / norm, 1.0)
    for g, o in zip(s["grads"], s["outs"]):
        o.copy_(g.float() * factor)
    return {"norm": norm, "grads": s["into"]}


def _own_embed(s):
    from paper_1702_07005_amd import features
    return features.embed(s["ids"], s["table"], scale=s["scale"], dtype=TYPES[s["case"]["out"]])


def _own_embed_grad(s):
    from paper_1702_07005_amd import features
    return features.embed_grad(s["ids"], s["grad"], s["case"]["rows"], scale=s["scale"], dtype=TYPES[s["case"]["table"]])


def _own_norm(s):
    from paper_1702_07005_amd import features
    y, mean, rstd = features.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS)
    return {"y": y, "mean": mean, "rstd": rstd}


def _own_norm_grad(s):
    from paper_1702_07005_amd import features
    dx, dw, db = features.layer_norm_grad(s["grad"], s["x"], s["mean"], s["rstd"], s["weight"])
    return {"x": dx, "weight": dw, "bias": db}


def _own_clip(s):
    from paper_1702_07005_amd import features
    return {"norm": features.clip_grads(s["grads"], s["limit"], out=s["outs"]), "grads": s["into"]}


_PLAIN = {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad,
          "clip": _plain_clip}
_OWN = {"embed": _own_embed, "embed_grad": _own_embed_grad, "norm": _own_norm, "norm_grad": _own_norm_grad,
        "clip": _own_clip}


# --------------------------------------------------------------------------- what it takes


def _distinct(tokens, rows, fields):
    """How many table rows are expected among the ids of ``_zipf_ids``: rank k of n has the share
    log(1 + 1/k) / log(n + 1) of its field's ids.  Ranks are taken in 400 ranges of equal ratio."""
    part, ids = rows // fields, 0.98 * tokens / fields
    total, k = 0.0, 1
    while k <= part:
        to = min(part + 1, max(k + 1, int(k * (part + 1) ** (1 / 400))))
        share = math.log(to / k) / math.log(part + 1) / (to - k)
        total += (to - k) * -math.expm1(ids * math.log1p(-min(share, 1 - 1e-12)))
        k = to
    return total * fields


def work(case):
    op = case["op"]
    if op == "embed":
        n, d = case["tokens"], case["dim"]
        seen = min(n, _distinct(n, case["rows"], case["fields"]))
        ids = n * (8 if case["wide_ids"] else 4)
        return {"bytes": ids + seen * d * BYTES[case["table"]] + n * d * BYTES[case["out"]], "flops": n * d}
    if op == "embed_grad":
        n, d = case["tokens"], case["dim"]
        ids = n * (8 if case["wide_ids"] else 4)
        return {"bytes": ids + n * d * BYTES[case["grad"]] + case["rows"] * d * BYTES[case["table"]], "flops": 2 * n * d}
    if op in ("norm", "norm_grad"):
        r, d, e, p = case["rows"], case["dim"], BYTES[case["type"]], BYTES[case["params"]]
        if op == "norm":
            return {"bytes": 2 * r * d * e + 8 * r + 2 * d * p, "flops": 7 * r * d}
        return {"bytes": 3 * r * d * e + 8 * r + 3 * d * p, "flops": 14 * r * d}
    n = sum(math.prod(s) for s in _clip_shapes(case))
    return {"bytes": n * (BYTES[case["type"]] + BYTES[case["out"]]) + 4, "flops": 3 * n}


# --------------------------------------------------------------------------- in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        table = torch.cat([s["table"].double() * s["scale"], torch.zeros(1, case["dim"], dtype=torch.float64, device="cuda")])
        return torch.nn.functional.one_hot(s["ids"].long() + 1, case["rows"] + 1).double()[:, 1:] @ table[:-1] \
            if case["tokens"] * case["rows"] <= 10_000_000 else table.index_select(0, s["ids"].long() % (case["rows"] + 1))
    if op == "embed_grad":
        # ids in order, running sums of their vectors, and each row's sum as the difference over its range
        order = torch.argsort(s["ids"].long(), stable=True)
        edges = torch.searchsorted(s["ids"].long()[order], torch.arange(case["rows"] + 1, device="cuda"))
        out = torch.empty(case["rows"], case["dim"], dtype=torch.float64, device="cuda")
        for c in range(0, case["dim"], 64):
            sums = torch.zeros(case["tokens"] + 1, min(64, case["dim"] - c), dtype=torch.float64, device="cuda")
            torch.cumsum(s["grad"][:, c:c + 64][order].double(), 0, out=sums[1:])
            out[:, c:c + 64] = (sums[edges[1:]] - sums[edges[:-1]]) * s["scale"]
        return out
    if op == "norm":
        x = s["x"].double()
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = 1 / torch.sqrt(var + EPS)
        y = torch.addcmul(s["bias"].double(), (x - mean[:, None]) * rstd[:, None], s["weight"].double())
        return {"y": y, "mean": mean, "rstd": rstd}
    if op == "norm_grad":
        # the derivative of y . grad, by way of d(x - mean), d(rstd) and d(mean)
        x, dy, rstd = s["x"].double(), s["grad"].double(), s["rstd"].double()
        centred = x - s["mean"].double()[:, None]
        dh = dy * s["weight"].double()
        drstd = (dh * centred).sum(1)
        dcentred = dh * rstd[:, None] - centred * (drstd * rstd ** 3 / case["dim"])[:, None]
        dx = dcentred - dcentred.sum(1, keepdim=True) / case["dim"]
        return {"x": dx, "weight": torch.matmul(rstd, dy * centred), "bias": dy.sum(0)}
    flat = s["flat"].double()
    norm = torch.linalg.vector_norm(flat)
    return {"norm": norm, "grads": flat.mul_((s["limit"] / norm).clamp(max=1.0))}
