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
