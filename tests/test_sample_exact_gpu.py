"""sample_logits at borders between tokens: minima, shares and uniform numbers so close
to a border that only weights of 64 bits tell its sides apart.  The same row goes through
every way that the kernels have (candidates of a short row, of a top-k, of slices;
histograms of one slice and of several) and has one answer: the definition's.

What is near: the borders are a few 10^-9 to 10^-8 of the weights' sum away, more than
V 2^-43 (the error of the sums, 4e-9 for the 32769 entries of a row padded to slices, of which
all but a few weigh nothing and are exact) and less than an exponent rounded to 32
bits is off by (2^-24 of it, 6e-8)."""
import numpy as np
import pytest

from oracle import more_serving as ms

torch = pytest.importorskip("torch")
from test_sample_gpu import BF16, F32, I32, INF, col, compare, logits, ta  # noqa: E402, F401

pytestmark = pytest.mark.gpu

# (logits, u, min_p, top_p, the token)
ROWS = [
    ((1.0409735, -0.9768613), 0.95, 0.13294299, None, 1),
    ((1.0, -0.75056094), 0.85202354, None, None, 1),
    ((1.0, -0.6177085), 0.83447886, None, None, 0),
    # weights that are 1.5, 1.1 and 0.2 10^-14 of themselves above min_p: what the series of a
    # histogram's weights may be off by
    ((0.91615325, -3.5037196), 0.99, 0.012035763, None, 1),
    ((3.5544543, -0.06282974), 0.98, 0.026855515, None, 1),
    ((1.0400137, -0.5636859), 0.9, 0.20115097, None, 1),
]
# (length the row is padded to with -inf, rows, top_k): how the kernels take it
WAYS = [(2, 1, None), (2, 5, 2), (1000, 1, None), (1025, 1, None), (2000, 3, None), (2000, 3, 2), (32768, 1, None),
        (100001, 1, None), (100001, 1, 2), (100001, 30, None), (100001, 30, 2), (40000, 130, None), (40000, 130, 2), (150001, 129, None),
        (150001, 129, 2)]


@pytest.mark.parametrize("V,B,k", WAYS, ids=str)
@pytest.mark.parametrize("row", ROWS, ids=["min_p", "u above", "u below", "1.5e-14", "1.1e-14", "2e-15"])
def test_one_answer_whichever_way_a_row_takes(ta, row, V, B, k):  # noqa: F811
    few, u, m, p, want = row
    first = np.float32(few)
    assert ms.sample(first, np.float32(u), min_p=0.0 if m is None else float(np.float32(m)))[0] == [want]
    some = lambda v, t=F32: None if v is None else col([v] * B, t)     # noqa: E731
    for at in {0, V - 2, (V - 2) // 2}:        # the two side by side, and far apart
        x = torch.full((B, V), -INF, device="cuda")
        x[:, at], x[:, at + 1] = float(first[0]), float(first[1])
        token, _ = ta.sample_logits(x, col([u] * B), None, some(k, I32), some(p), some(m))
        assert (token == at + want).all(), (at, token.tolist())
    x = torch.full((B, V), -INF, device="cuda")
    x[:, 0], x[:, V - 1] = float(first[0]), float(first[1])
    token, _ = ta.sample_logits(x, col([u] * B), None, some(k, I32), some(p), some(m))
    assert (token == (V - 1 if want else 0)).all()


def beside(c):
    """The 32-bit numbers below and above each border c."""
    lo = c.astype(np.float32)
    lo = np.where(lo > c, np.nextafter(lo, np.float32(0)), lo)
    return np.concatenate([lo, np.nextafter(lo, np.float32(1))])


@pytest.mark.parametrize("T", [None, 0.7])
@pytest.mark.parametrize("V", [2, 3, 17, 300, 1024])
def test_numbers_beside_the_borders(ta, V, T):  # noqa: F811
    """u, the 32-bit numbers on both sides of the share of the tokens up to some index; the
    same shares as top_p, and weights as min_p, in rows whose order is that of the indexes,
    so that the last token that stays is the one taken."""
    n = 64
    x, _, g = logits(1, V, F32, V, (2.0, 2.0))
    pick = torch.randint(0, V - 1, (n // 2,), generator=g).numpy()
    temperature = None if T is None else [T] * n

    def both_ways(row, u, p=None, m=None):
        # Both answers count where a 32-bit number is within V 2^-43 of the border (1.2e-10 at
        # most): for shares, 2^-26 apart and more, one in a hundred; for weights of 0.02 and more,
        # 2^-29 apart, one in sixteen
        padded = torch.full((n, 1500), -INF, device="cuda")
        padded[:, :V] = row
        for y in (row.expand(n, V).contiguous(), padded):
            compare(ta, y, u, temperature, None, p, m, unclear=n // 4)

    def weights(row):
        row = row.double().cpu().numpy()
        return np.exp((row - row.max()) / (1.0 if T is None else float(np.float32(T))))

    w = weights(x[0])
    both_ways(x, beside((np.cumsum(w) / w.sum())[pick]))
    x = x.sort(descending=True).values
    w = weights(x[0])
    last = [1 - 2.0 ** -24] * n
    both_ways(x, last, beside((np.cumsum(w) / w.sum())[pick]))
    large = max(2, int((w >= 0.02).sum()))
    both_ways(x, last, None, beside(w[1 + pick % (large - 1)]))
