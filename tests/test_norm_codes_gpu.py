"""The codes and scales of the root-mean-square norm in 8 bits, bit by bit, against the 32-bit computation that the C header
states, on the CPU: with the rows' factors given, every later rounding is one of a product, a quotient or a conversion."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_1702_07005_amd import features  # noqa: E402

DEV = "cuda"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
E4M3 = torch.float8_e4m3fn


def _stated(h, weight, rstd, group):
    """(codes, scales) in 32 bits; torch divides on the CPU as IEEE 754 does."""
    y = h.float() * rstd[:, None]
    if weight is not None:
        y = y * weight.float()
    rows, dim = y.shape
    g = group or dim
    c = torch.tensor(1.0, dtype=F32) / torch.tensor(448.0, dtype=F32)
    top = torch.nn.functional.pad(y, (0, -dim % g)).view(rows, -1, g).abs().nan_to_num(0.0, float("inf")).amax(2)
    scale = (top * c).clamp(min=2.0 ** -126)
    codes = (y / scale.repeat_interleave(g, 1)[:, :dim]).to(E4M3)
    return codes.view(torch.uint8), scale if group else scale[:, 0]


def _same(x, weight, group, **kw):
    q, scale, rstd, _ = features.rms_norm_8bit(x.to(DEV), None if weight is None else weight.to(DEV), group=group, **kw)
    codes, scales = _stated(x, weight, rstd.cpu(), group)
    assert torch.equal(scale.cpu(), scales)
    got = q.view(torch.uint8).cpu()
    nan = (got & 0x7F) == 0x7F  # either sign
    assert torch.equal(nan, (codes & 0x7F) == 0x7F)
    bad = (got != codes) & ~nan
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} codes differ"


# Every group of lanes, rows that are read again, and both sides of a vector; 16-bit factors make quotients that lie in the
# middle between two codes, or next to it.
@pytest.mark.parametrize("x,p", [(F32, F32), (BF16, BF16), (F16, F32)], ids=str)
@pytest.mark.parametrize("dim", [3, 30, 60, 250, 500, 1500, 2049, 2500, 4096, 6150, 8193, 12_300, 16_384, 20_001, 40_000])
def test_codes_are_those_of_the_stated_roundings(dim, x, p):
    g = torch.Generator().manual_seed(dim)
    rows = min(4096, 2_000_000 // dim)
    h = ((torch.randn(rows, dim, generator=g) + 0.1) * (0.1 + 2 * torch.rand(rows, 1, generator=g))).to(x)
    w = (1 + 0.3 * torch.randn(dim, generator=g)).to(p)
    for group in (None, 32, 64, 128):
        _same(h, w, group)
    _same(h, None, None)


# Scales too small for a remainder in 32 bits, the least one, an infinite one, and rows of zeros and NaN.
@pytest.mark.parametrize("group", [None, 32])
@pytest.mark.parametrize("dim", [5, 96, 1000, 4100, 17_000])
def test_codes_of_rows_far_from_one(dim, group):
    g = torch.Generator().manual_seed(dim)
    sizes = torch.tensor([2.0 ** -k for k in range(0, 149, 4)] + [0.0, 2.0 ** 30, 2.0 ** 60])
    h = torch.randn(sizes.numel(), dim, generator=g) * sizes[:, None]
    w = 1 + 0.3 * torch.randn(dim, generator=g)
    _same(h, w, group)  # 1e-6 under the root leaves small rows small
    _same(h, None, group, eps=1.0)
    bad = h.clone()
    bad[3, dim // 2], bad[5, 0], bad[7, dim - 1] = float("nan"), float("inf"), -float("inf")
    _same(bad, w, group)
    w[dim // 3] = float("inf")
    _same(h, w, group)
    w[dim // 2] = float("nan")
    _same(h, w, group)
