"""What the root-mean-square norm returns for its gradient: h, the values that it normalised."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_1702_07005_amd import features  # noqa: E402

DEV = "cuda"


@pytest.mark.parametrize("rows", [1, 9])
@pytest.mark.parametrize("dim", [7, 96, 5000, 20_000])
def test_kept_values_are_those_before_the_call(rows, dim):
    g = torch.Generator().manual_seed(dim)
    x, res = torch.randn(rows, dim, generator=g).to(DEV), torch.randn(rows, dim, generator=g).to(DEV)
    w = torch.ones(dim, device=DEV)
    # in x's place nothing holds them any more
    for same in (lambda t: t, lambda t: t.view(rows, dim), lambda t: t[:, :]):
        place = x.clone()
        y, rstd, h = features.rms_norm(place, w, out=same(place))
        assert h is None and torch.equal(y, features.rms_norm(x, w)[0])
    # elsewhere x does, and with a residual the sum
    y, rstd, h = features.rms_norm(x, w, out=torch.empty_like(x))
    assert h is x
    for out, total in ((0, 1), (1, 0)):
        place = [x.clone(), res.clone()]
        h = features.rms_norm(place[0], w, place[1], out=place[out], sum_out=place[total])[2]
        assert h is place[total] and torch.equal(h, x + res)
    place = x.clone()
    h = features.rms_norm(place, w, res, out=place)[2]
    assert torch.equal(h, x + res)
    # 8 bits have memory of their own
    assert features.rms_norm_8bit(x, w)[3] is x


def test_kept_values_without_rows():
    x = torch.empty(0, 33, device=DEV)
    assert features.rms_norm(x, out=torch.empty_like(x))[2] is x


# The calls are outside autograd: no result requires gradients, the caller's own x among them.
@pytest.mark.parametrize("call", [features.rms_norm, features.rms_norm_8bit], ids=["rms_norm", "rms_norm_8bit"])
def test_no_result_requires_gradients(call):
    leaf = torch.randn(6, 64, device=DEV, requires_grad=True)
    for x in (leaf, leaf * 2):
        for res in (None, leaf):
            results = call(x, leaf[0], res)
            assert not any(t.requires_grad for t in results)
            h = results[-1]
            assert torch.equal(h, x.detach() if res is None else x.detach() + leaf.detach())
            assert res is not None or (h.data_ptr() == x.data_ptr() and h._version == x._version)
        with torch.no_grad():
            assert not call(x)[-1].requires_grad
    plain = leaf.detach()
    assert call(plain)[-1] is plain
