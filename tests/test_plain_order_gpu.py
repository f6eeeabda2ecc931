"""The plain kernels with few coordinates in flight, and the pipelined one with a workgroup for each of a given number, take them
in the order of the permutation, also where one workgroup draws all the long segments."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import numpy as np  # noqa: E402

from oracle import oracle as orc  # noqa: E402
from paper_1702_07005_amd import scd, synth  # noqa: E402


# Columns of ones on supports of their own, each twice: the one that comes first takes the whole of the labels there and leaves
# the other nothing.  At a fixed stride one of four workgroups would draw all the first ones, which are long (explicit zeros),
# and the others would long have reached the second ones, 50 turns later in the permutation.
@pytest.mark.parametrize("kernel,lanes", [("block", 256), ("mixed", 64), ("pipelined", 256)])
def test_kernels_keep_the_order(kernel, lanes):
    turn = 256 // lanes                 # positions that a workgroup takes at a time
    pairs, apart, short, zeros, W = 200, 50, 300, 20_000, 4
    n = W * turn * (pairs + apart + 2)
    seed = 3
    perm = scd.permutation(seed, 0, n).cpu().numpy().astype(np.int64)
    first = [W * turn * i for i in range(pairs)]
    second = [W * turn * (i + apart) + 2 * turn for i in range(pairs)]
    L = pairs * short + zeros
    support = {}
    for i in range(pairs):
        here = np.arange(i * short, (i + 1) * short)
        support[perm[first[i]]] = (np.concatenate([here, np.arange(pairs * short, L)]), np.concatenate([np.ones(short), np.zeros(zeros)]))
        support[perm[second[i]]] = (here, np.ones(short))
    rest = (np.arange(L - short, L), np.ones(short))  # where the labels are 0
    columns = [support.get(c, rest) for c in range(n)]
    ptr = np.concatenate([[0], np.cumsum([len(i) for i, _ in columns])])
    idx, val = np.concatenate([i for i, _ in columns]), np.concatenate([v for _, v in columns])
    y = np.concatenate([np.ones(pairs * short), np.zeros(zeros)])
    dev = [torch.from_numpy(np.ascontiguousarray(t)).to("cuda") for t in (ptr.astype(np.int64), idx.astype(np.int32), val.astype(np.float32), y.astype(np.float32))]
    s = scd.Solver(L, n, *dev, 1e-9, "ridge_primal")
    s.set_option("pipeline", int(kernel == "pipelined"))
    s.set_option("group", lanes)
    s.set_option("window", W * turn)
    info = s.info()
    print(f"{kernel}: kernel {info['kernel']} window {info['window']} of {n}", flush=True)
    assert info["kernel"] == kernel and info["window"] == W * turn
    for _ in range(2):  # the queue starts from 0 in every epoch
        s.set_state(torch.zeros(n, device="cuda"), torch.zeros(L, device="cuda"), 0)
        s.epochs(seed, 1)
        model = s.get_state()[0].double().cpu().numpy()
        a, b = model[perm[first]], model[perm[second]]
        late = int((b > a).sum())
        assert late == 0, f"{late} of {pairs} pairs the wrong way round"
        assert np.abs(a - 1).max() < 1e-3 and np.abs(b).max() < 1e-3
    s.close()


# Twice the sequential algorithm's gap, in the default plan of the plain kernels, over runs enough to tell one run in thirty.
@pytest.mark.parametrize("seed", [0, 1, 2])
def test_block_kernel_stays_near_the_sequential_gap(seed):
    p = synth.make("text_svm", n_rows=3_500, n_cols=166_000, row_nnz=370)
    model, shared, curve = np.zeros(p.C), np.zeros(p.L), []
    for e in range(8):
        orc.epochs(p.form, p.n_rows, p.n_cols, p.ptr, p.idx, p.val, p.y, p.lam, seed, e, 1, model, shared)
        curve.append(orc.objectives(p.form, p.n_rows, p.n_cols, p.ptr, p.idx, p.val, p.y, p.lam, model, shared)[2])
    worst = []
    for _ in range(20):
        s = scd.solver_for(p)
        s.set_option("pipeline", 0)
        assert s.info()["kernel"] == "block"
        P0, _ = s.objective()
        ratios = []
        for Gr in curve:
            s.epochs(seed, 1)
            ratios.append((s.duality_gap() - 1e-6 * abs(P0)) / Gr)
        worst.append(max(ratios))
        s.close()
    print(f"seed {seed}: worst ratios {min(worst):.2f} to {max(worst):.2f}", flush=True)
    assert max(worst) <= 2.0
