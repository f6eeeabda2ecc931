"""The operators of learned features on the GPU, at sizes chosen by the code that they reach: every sort of the
lookup gradient, every join of its sums, loads and stores past the caches, second turns of the row loops, whole chunks
of the clipping.  Outputs hold NaN before the call, so that an element that is not written shows."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import _features_oracle as fo  # noqa: E402
from paper_1702_07005_amd import features  # noqa: E402

DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _give_back_memory():
    yield
    torch.cuda.empty_cache()


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _nan(*shape, dtype=torch.float32):
    return torch.full(shape, float("nan"), dtype=dtype, device=DEV)


# ---------------------------------------------------------------- lookup


def test_embed_more_tokens_than_one_launch_takes():
    # Rows of 256 lanes: a launch takes 67,108,860 tokens at four for each workgroup.
    n, rows, dim = 67_108_860 + 1_001, 2_000, 1025
    if torch.cuda.mem_get_info()[0] < 2 * n * dim + (8 << 30):
        pytest.skip("needs 146 GB of GPU memory")
    g = torch.Generator(device=DEV).manual_seed(1)
    table = torch.randn(rows, dim, generator=g, device=DEV).bfloat16()
    t = torch.randint(-1, rows, (n,), generator=g, device=DEV, dtype=torch.int32)
    out = features.embed(t, table)
    full = torch.cat([table, torch.zeros(1, dim, dtype=table.dtype, device=DEV)])  # -1 is its last row
    for at in range(0, n, 1 << 20):
        assert torch.equal(out[at:at + (1 << 20)], full[t[at:at + (1 << 20)].long()]), at


# ---------------------------------------------------------------- zeros of the lookup gradient


# Tables whose zeros, shared out among workgroups in whole 64-byte lines, leave a remainder: the last bytes of each
# launch's part lie in rows without tokens.
@pytest.mark.parametrize("n,rows,dim,dtype,spare", [
    (2_000, 52_000, 300, torch.float32, (25_999, 51_999)), (20_000, 52_000, 300, torch.float32, (25_999, 51_999)),
    (2_000, 57_000, 255, torch.float32, (28_499, 56_999)), (100_000, 3_000, 333, torch.bfloat16, (499, 1_499, 1_999, 2_999))])
def test_embed_grad_zeros_reach_the_end_of_every_part(n, rows, dim, dtype, spare):
    g = _gen(n + rows)
    t = torch.randint(0, rows, (n,), generator=g)
    for r in spare:
        t[t == r] = 0
    d = torch.randn(n, dim, generator=g).to(dtype)
    out = features.embed_grad(t.to(DEV), d.to(DEV), rows, out=_nan(rows, dim, dtype=dtype))
    fo.close(out, fo.embed_grad(t, d, rows, 1.0, dtype), "embed_grad")


# ---------------------------------------------------------------- beside autograd


def _writes(x, y, grads):
    """Calls that write to x (out, accumulation, in place) or to the gradients."""
    ids = torch.arange(6, device=DEV)
    n = x.shape[1]
    _, mean, rstd = features.layer_norm(y)
    yield x, lambda: features.embed(ids, y, out=x)
    yield x, lambda: features.embed_grad(ids, y, 6, out=x)
    yield x, lambda: features.embed_grad(ids, y, 6, out=x, accumulate=True)
    yield x, lambda: features.layer_norm(y, torch.ones(n, device=DEV), out=x)
    yield x, lambda: features.layer_norm(x, out=x)
    yield x, lambda: features.layer_norm_grad(y, y, mean, rstd, out=x)
    yield grads[1], lambda: features.clip_grads(grads, 1e-3)
    yield x, lambda: features.clip_grads(grads[:1], 1e-3, out=[x])


def _six():
    return torch.randn(6, 8, device=DEV)


def test_writes_count_as_in_place_operations():
    x, y, grads = _six(), _six(), [_six(), _six()]
    for k, (to, call) in enumerate(_writes(x, y, grads)):
        before, others, view = to._version, (y._version, grads[0]._version), to[1:3]
        call()
        assert to._version > before and view._version == to._version, k
        if k != 6:
            assert (y._version, grads[0]._version) == others, k
    before = [g._version for g in grads]
    features.grad_norm(grads)
    assert [g._version for g in grads] == before
    with torch.inference_mode():
        z = _six()
    for to, call in _writes(z, y, [z, z.clone()]):
        call()


def test_autograd_notices_overwritten_values():
    for k in range(8):
        x, grads = _six(), [_six(), _six()]
        to, call = list(_writes(x, _six(), grads))[k]
        p = _six().requires_grad_()
        loss = (p * to).sum()
        call()
        with pytest.raises(RuntimeError, match="in-?place"):
            loss.backward()


def test_tensors_that_require_gradients():
    table = _six().requires_grad_()
    got = features.embed(torch.arange(6, device=DEV), table)
    assert not got.requires_grad and torch.equal(got, table)
    for k in range(8):
        for leaf in (True, False):
            x = _six().requires_grad_() if leaf else _six().requires_grad_() * 2
            grads = [_six(), _six().requires_grad_() if leaf else _six().requires_grad_() * 2]
            to, call = list(_writes(x, _six(), grads))[k]
            before = to.detach().clone()
            with pytest.raises(ValueError, match="requires gradients"):
                call()
            assert torch.equal(to, before)
            with torch.no_grad():
                call()
            assert not torch.equal(to, before), k
