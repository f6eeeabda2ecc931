"""A ridge read-out on learned features: the solver fits the read-out, its gradient trains the table below it.

Documents are lists of term ids (Zipf's law, of unequal lengths, the rest of a row padded with -1), each with a
label that its terms' hidden weights give.  A document's features are the mean of its terms' normalised
vectors.  An iteration looks the terms up, normalises their vectors, fits the read-out by coordinate descent from
where it stood, and takes one step of gradient descent on the table and the norm's parameters, clipped by the
norm of all three gradients together:

    python examples/learned_features.py [--iterations 12] [--documents 8192]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_1702_07005_amd import features, scd


def documents(n, length, terms, seed):
    """Ids [n, length], -1 where a document has ended, and labels of zero mean and unit variance."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rank = torch.expm1(torch.rand(n, length, device="cuda", generator=g) * torch.log(torch.tensor(terms + 1.0))).long()
    ids = rank.clamp_(max=terms - 1)
    ends = torch.randint(length // 4, length + 1, (n, 1), device="cuda", generator=g)
    there = torch.arange(length, device="cuda") < ends
    hidden = torch.randn(terms, device="cuda", generator=g)
    label = (hidden[ids] * there).sum(1) / ends[:, 0]
    return ids.masked_fill_(~there, -1), (label - label.mean()) / label.std()


def train(iterations=12, n=8192, length=48, terms=3000, dim=64, lam=1e-3, rate=20.0, max_norm=0.2, seed=0, report=None):
    """The primal objective of the fitted read-out in each iteration."""
    ids, label = documents(n, length, terms, seed)
    there = (ids >= 0).unsqueeze(2)
    share = there / there.sum(1, keepdim=True)  # of each place in its document's features
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    table = torch.randn(terms, dim, device="cuda", generator=g) * dim ** -0.5
    weight, bias = torch.ones(dim, device="cuda"), torch.zeros(dim, device="cuda")
    scale = dim ** 0.5
    # the features as a matrix by columns: every entry is there
    ptr = torch.arange(dim + 1, device="cuda") * n
    idx = torch.arange(n, dtype=torch.int32, device="cuda").repeat(dim)
    readout = torch.zeros(dim, device="cuda")
    objectives = []
    for k in range(iterations):
        x = features.embed(ids, table, scale=scale)
        y, mean, rstd = features.layer_norm(x, weight, bias)
        docs = (y * share).sum(1)
        with scd.Solver(n, dim, ptr, idx, docs.t().contiguous().view(-1), label, lam, "ridge_primal") as solver:
            solver.set_state(readout, docs @ readout)
            solver.epochs(seed + k, 10)
            primal, dual = solver.objective()
            readout, shared, _ = solver.get_state()
        objectives.append(primal)
        # P = |docs readout - label|^2 / (2 n) + lam / 2 |readout|^2, with respect to docs, then to the places' vectors
        ddocs = torch.outer(shared - label, readout) / n
        dy = share * ddocs.unsqueeze(1)
        dx, dweight, dbias = features.layer_norm_grad(dy, x, mean, rstd, weight)
        dtable = features.embed_grad(ids, dx, terms, scale=scale)
        grads = [dtable, dweight, dbias]
        norm = features.clip_grads(grads, max_norm)
        for p, d in zip((table, weight, bias), grads):
            p.sub_(d, alpha=rate if p is table else 1.0)
        if report:
            report(f"iteration {k}: primal objective {primal:.6f}, gap {primal - dual:.1e}, gradient norm {float(norm):.4f}")
    return objectives


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--iterations", type=int, default=12)
    ap.add_argument("--documents", type=int, default=8192)
    a = ap.parse_args()
    train(iterations=a.iterations, n=a.documents, report=lambda line: print(line, flush=True))
