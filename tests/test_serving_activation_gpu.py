"""silu and the tanh gelu of gemm_bf16_epilogue with an fp32 C, relative to the value, over
the whole range of the exponential.

Tolerance: the hardware's exponential and reciprocal are off by an ulp each (2^-23), the
correction of the exponent, the sum and the product with x by half an ulp each (2^-24): 7
2^-24, below 2^-21; ln 2 as one fp32 number is off by 2^-28.4 of itself, times an exponent of
at most 128: 2^-22 |x| / 87.  Beyond e^88.72 the sum 1 + e^-x is infinite and the result 0:
88.73 2^-128 is below 2^-121.

The argument is a sum of two products.  Where it has more than 24 bits fp32 cannot hold it:
it is off by up to 2^-23 of itself (an ulp, however the sum is rounded), and silu, whose
slope is below (1 + |x|) silu(x) / |x|, by (1 + |x|) 2^-23 of its value."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def ta():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2504_17577_amd import tileattn
    tileattn.lib()
    return tileattn


def arguments(lo, hi):
    """Every bf16 number of that size, and its negative, with a second bf16 number added
    that fills the bits below; which of the sums fp32 holds exactly."""
    x = torch.tensor([lo, hi]).to(BF16).view(torch.int16)
    x = torch.arange(int(x[0]), int(x[1]) + 1, dtype=torch.int32).to(torch.int16).view(BF16)
    x = torch.cat([x, -x])
    low = (x.float() * torch.rand(len(x), generator=torch.Generator().manual_seed(1)) / 512).to(BF16)
    a = torch.zeros(len(x), 8, dtype=BF16)
    a[:, 0], a[:, 1] = x, low
    b = torch.zeros(8, 8, dtype=BF16)
    b[:2] = 1
    y = x.double() + low.double()
    held = y == y.float().double()
    assert held.sum() > len(y) / 3
    return a, b, y, held


@pytest.mark.parametrize("rows", [1 << 20, 64, 7], ids=["tiled", "few64", "few7"])
@pytest.mark.parametrize("lo,hi", [(2.0 ** -20, 60.0), (60.0, 120.0)])
def test_silu_relative_to_its_value(ta, lo, hi, rows):
    a, b, y, held = arguments(lo, hi)
    a, b = a.cuda(), b.cuda()
    parts = a.split(rows) if len(a) / rows < 20 else [a[i:i + rows] for i in range(0, len(a) - rows, len(a) // 20)] + [a[-rows:]]
    at = torch.arange(len(a)).split(rows) if len(a) / rows < 20 else \
        [torch.arange(i, i + rows) for i in range(0, len(a) - rows, len(a) // 20)] + [torch.arange(len(a) - rows, len(a))]
    for p, i in zip(parts, at):
        got = ta.gemm_bf16_epilogue(p.contiguous(), b, activation="silu")[:, 0].double().cpu()
        want = y[i] / (1 + torch.exp(-y[i]))
        tol = want.abs() * (2.0 ** -21 + 2.0 ** -22 * y[i].abs() / 87 + ~held[i] * (1 + y[i].abs()) * 2.0 ** -23) + 2.0 ** -121
        over = ((got - want).abs() / tol).max()
        assert over <= 1, f"{float(over):.2f} of the tolerance"


def test_tanh_gelu_relative_to_its_value(ta):
    """As silu of u = 2 sqrt(2/pi) (x + 0.044715 x^3), times x / u; u in fp32 is off by 7 2^-24
    of itself (four products and a sum, two constants), and by 3 times what x is off by
    where fp32 does not hold x."""
    a, b, x, held = arguments(2.0 ** -20, 8.0)
    got = ta.gemm_bf16_epilogue(a.cuda(), b.cuda(), activation="gelu_tanh")[:, 0].double().cpu()
    u = 2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)
    want = x / (1 + torch.exp(-u))
    tol = want.abs() * (2.0 ** -21 + 2.0 ** -22 * u.abs() / 87 + 7 * 2.0 ** -24 * u.abs() + ~held * (1 + 3 * u.abs()) * 2.0 ** -23) + 2.0 ** -121
    assert ((got - want).abs() <= tol).all()
