"""GPU parity of sample_logits against the float64 oracle.  A token has to be
the oracle's, or one of its answers for sums of weights that are off by V 2^-43 (the
weights are whole multiples of 2^-43, V of them rounded by half of one, and the oracle's
sums by less); rows on borders on purpose have closed forms.  logp's tolerance: its sum's terms in
fp32 by the hardware's exponential (2^-23 and the exponent's rounding, |d| 2^-24 of a
term e^-d, at most 2^-25.4 where they are weighed), up to 256 of them added in fp32 per
thread (2^-24 each at most), then half a step of the result: |dlogp| <= 260 2^-24 + 2^-24 |logp|."""
import numpy as np
import pytest

from oracle import more_serving as ms

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ta():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2504_17577_amd import tileattn
    tileattn.lib()
    return tileattn


def col(x, dtype=F32):
    return None if x is None else torch.as_tensor(x, dtype=dtype).cuda()


def compare(ta, x, u, T=None, k=None, p=None, m=None, unclear=1):
    """sample_logits(x, ..) row by row against the oracle; at most `unclear` rows may have
    more than one answer."""
    B, V = x.shape
    token, logp = ta.sample_logits(x, col(u), col(T), col(k, I32), col(p), col(m))
    token, logp, rows = token.cpu().numpy(), logp.cpu().numpy(), x.double().cpu().numpy()
    f32 = lambda v, i, d: d if v is None else float(np.float32(v[i]))    # noqa: E731
    more = 0
    for b in range(B):
        want, lps = ms.sample(rows[b], f32(u, b, 0), f32(T, b, 1.0), 0 if k is None else int(k[b]), f32(p, b, INF),
                              f32(m, b, 0.0), V * 2.0 ** -43)
        assert token[b] in want, (b, token[b], want)
        more += len(want) > 1
        if want == [-1]:
            assert np.isnan(logp[b])
        else:
            lp = lps[want.index(token[b])]
            assert abs(logp[b] - lp) <= 260 * 2.0 ** -24 + 2.0 ** -24 * abs(lp), (b, logp[b], lp)
    assert more <= unclear, more
    return token, logp


def logits(B, V, dtype, seed, spread=(1.0, 4.0)):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(B, V, generator=g) * torch.linspace(*spread, B)[:, None]
    return x.to(dtype).cuda(), torch.rand(B, generator=g).numpy(), g


FILTERS = [(None, None, None), (50, None, None), (None, 0.9, None), (None, None, 0.05), (40, 0.8, None), (3000, 0.95, 0.001),
           (700, None, None), (1, None, None), (20, 0.97, 0.02)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("B,V", [(5, 1), (7, 2), (6, 9), (9, 100), (5, 1023), (4, 1025), (130, 515), (5, 4099), (6, 32000), (6, 32768),
                                 (7, 32769), (4, 70001), (3, 128001), (1, 200000), (130, 40000)])
def test_against_oracle(ta, B, V, dtype):
    for i, (k, p, m) in enumerate(FILTERS):
        x, u, g = logits(B, V, dtype, V + i)
        T = torch.rand(B, generator=g).numpy() + 0.4
        if B > 3:
            T[B // 2] = 0
        some = lambda v: None if v is None else [v] * B     # noqa: E731
        compare(ta, x, u, T, some(k), some(p), some(m))


def test_a_wish_for_each_row(ta):
    """Filters, temperatures and kinds of rows that differ from row to row, with all of
    their special values."""
    B, V = 96, 50001
    x, u, g = logits(B, V, F32, 1, (0.05, 8.0))
    pick = lambda *v: np.array(v, np.float64)[torch.randint(0, len(v), (B,), generator=g).numpy()]   # noqa: E731
    k = pick(0, -3, 1, 2, 63, 64, 300, 2000, V - 1, V, V + 1, 2 ** 31 - 1).astype(np.int64)
    p = pick(0.0, -1.0, 0.3, 0.9, 0.999, 1.0, 2.0, NAN, 1e-8)
    m = pick(0.0, -1.0, 1e-5, 0.1, 0.9999, 1.5, NAN)
    T = pick(0.0, -2.0, NAN, 0.1, 1.0, 3.0, INF, 1e-38, 1e30)
    compare(ta, x, u, T, k, p, m)
    compare(ta, x.to(BF16), u, T, k, p, m)
    compare(ta, x[:, :3000].contiguous(), u, T, np.minimum(k, 2 ** 20), p, m)


@pytest.mark.parametrize("B,V,dtype", [(2, 1 << 20, F32), (2, 1 << 20, BF16), (131, 150001, F32), (129, 139264, BF16), (128, 139265, BF16)])
def test_largest_rows(ta, B, V, dtype):
    """Rows that have to be cut in slices however many there are; the largest allowed.  The
    oracle takes a few of them."""
    for k, p, m in ((50, 0.9, None), (None, 0.9, None), (2500, None, 0.001)):
        x, u, _ = logits(B, V, dtype, V + (k or 0))
        some = lambda v, t=F32: None if v is None else col([v] * B, t)     # noqa: E731
        token, logp = ta.sample_logits(x, col(u), None, some(k, I32), some(p), some(m))
        for b in (0, B // 2, B - 1):
            args = [0 if k is None else k] + [d if v is None else float(np.float32(v)) for v, d in ((p, INF), (m, 0.0))]
            want, lps = ms.sample(x[b].double().cpu().numpy(), float(u[b]), 1.0, *args, V * 2.0 ** -43)
            assert int(token[b]) in want and len(want) <= 2
            lp = lps[want.index(int(token[b]))]
            assert abs(float(logp[b]) - lp) <= 260 * 2.0 ** -24 + 2.0 ** -24 * abs(lp)


@pytest.mark.parametrize("V", [1000, 30000, 100001])
def test_masked_rows(ta, V):
    """-inf in all but a few places, in whole slices, and everywhere; NaN and +inf."""
    B = 12
    x, u, g = logits(B, V, F32, V)
    x[0, 1:] = -INF
    x[1, :V - 1] = -INF
    x[2, 7:V - 5] = -INF
    x[3] = -INF
    x[4, V // 2] = NAN
    x[5, V - 1] = INF
    x[6, :V - 3] = -INF
    x[6, V - 2] = NAN
    x[7] = -INF
    x[7, V - 1] = NAN
    x[8] = NAN
    x[9, ::2] = -INF
    x[10, 3], x[10, 4] = INF, -INF
    for k, p, m in FILTERS:
        some = lambda v: None if v is None else [v] * B     # noqa: E731
        token, logp = compare(ta, x, u, None, some(k), some(p), some(m))
        assert token[0] == 0 and token[1] == V - 1 and (logp[:2] == 0).all()
        assert (token[[3, 4, 5, 6, 7, 8, 10]] == -1).all()
    token, _ = ta.sample_logits(x, col(u), col([0.0] * B))
    assert token.tolist()[3] == -1 and token.tolist()[4] == -1 and token.tolist()[1] == V - 1


@pytest.mark.parametrize("V", [64, 5000, 40000, 131072])
def test_ties(ta, V):
    """Equal logits: the order is by index, every sum exact."""
    B = 8
    u = np.array([0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24, 0.5, 0.999, 0.0])
    x = torch.full((B, V), 3.25, device="cuda")
    token, logp = (t.cpu().numpy() for t in ta.sample_logits(x, col(u)))
    np.testing.assert_array_equal(token, np.floor(u.astype(np.float32) * np.float64(V)).astype(int))
    assert (np.abs(logp + np.log(V)) <= 260 * 2.0 ** -24 + 2.0 ** -24 * np.log(V)).all()
    for k in (1, 40, V // 4, V - 1):        # the first k by index
        token, _ = ta.sample_logits(x, col(u), top_k=col([k] * B, I32))
        np.testing.assert_array_equal(token.cpu().numpy(), np.floor(u.astype(np.float32) * np.float64(k)).astype(int))
    for p in (0.25, 0.5, 1.0):              # before_i = i < p V
        token, _ = ta.sample_logits(x, col(u), top_p=col([p] * B))
        np.testing.assert_array_equal(token.cpu().numpy(), np.floor(u.astype(np.float32) * np.ceil(p * V)).astype(int))
    token, _ = ta.sample_logits(x, col(u), min_p=col([1.0] * B))
    np.testing.assert_array_equal(token.cpu().numpy(), np.floor(u.astype(np.float32) * np.float64(V)).astype(int))
    token, _ = ta.sample_logits(x, col(u), col([0.0] * B))
    assert (token == 0).all()
    # -0 is 0; a row of two values, many of each, the border among the lower ones
    x[:, ::2], x[:, 1::2] = 0.0, -0.0
    token, _ = ta.sample_logits(x, col(u), top_k=col([V // 2] * B, I32))
    np.testing.assert_array_equal(token.cpu().numpy(), np.floor(u.astype(np.float32) * np.float64(V // 2)).astype(int))
    x[:, 1::2] = -np.log(2.0)
    for p in (0.75, 0.9):
        compare(ta, x, u, None, None, [p] * B, unclear=B)
    k = [V // 2 + V // 4] * B
    compare(ta, x, u, None, k, None)


@pytest.mark.parametrize("V", [9000, 60000])
def test_narrow_and_ordered_rows(ta, V):
    """All of a row in one bucket, with thousands of different logits; rows in falling and
    rising order, of which a few threads would have all candidates; a few distinct values."""
    B = 8
    x, u, g = logits(B, V, F32, V, (1e-6, 1e-3))
    x[3] = x[3].sort().values
    x[4], x[5] = torch.linspace(5, -5, V), torch.linspace(-5, 5, V)
    x[6] = (torch.randn(V, generator=g) * 2).round()
    x[7] = torch.where(torch.arange(V) < V // 2, 1.0, 1.0 + 2.0 ** -20).roll(17)
    for k, p, m in FILTERS + [(V // 3, 0.9, None), (V // 3, None, None), (None, 0.3, None), (None, None, 0.9999)]:
        some = lambda v: None if v is None else [v] * B     # noqa: E731
        compare(ta, x, u, None, some(k), some(p), some(m))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V", [77, 33001])
def test_rows_of_a_wider_tensor(ta, V, dtype):
    """Rows at every offset from a 16-byte line, NaN before and behind them."""
    for shift in range(8):
        x = torch.full((5, V + 24), NAN, dtype=dtype, device="cuda")
        y, u, _ = logits(5, V, dtype, shift)
        x[:, shift:shift + V] = y
        compare(ta, x[:, shift:shift + V], u, None, [30] * 5, [0.9] * 5)
        compare(ta, x[:, shift:shift + V], u, None, None, [0.9] * 5)


def test_uniform_numbers_from_end_to_end(ta):
    """Over many u the tokens come as often as their weights say, each where its share
    begins: against the cumulative sums."""
    V, n = 37, 4096
    x, _, _ = logits(1, V, F32, 5, (1.5, 1.5))
    u = (np.arange(n) + 0.5) / n
    token, logp = ta.sample_logits(x.expand(n, V).contiguous(), col(u))
    w = np.exp(x[0].double().cpu().numpy())
    want = np.searchsorted(np.cumsum(w) / w.sum(), u.astype(np.float32), side="right")
    np.testing.assert_array_equal(token.cpu().numpy(), want)
    token, _ = ta.sample_logits(x.expand(4, V), col([-1.0, NAN, 1.0, INF]))       # outside: the ends
    assert token.tolist() == [0, 0, V - 1, V - 1]


def test_rows_past_2_gib(ta):
    B, V, stride = 3, 40000, 1 << 30
    big = torch.empty((B - 1) * stride + V, dtype=BF16, device="cuda")
    rows = big.as_strided((B, V), (stride, 1))
    x, u, _ = logits(B, V, BF16, 6)
    rows.copy_(x)
    for k in (None, [50] * B):
        kk = col(k, I32)
        a, b = ta.sample_logits(rows, col(u), top_k=kk), ta.sample_logits(x, col(u), top_k=kk)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("B,V", [(3, 500), (3, 60000), (140, 40000)])
def test_captured_and_on_a_side_stream(ta, B, V):
    """One capture serves new logits, numbers and wishes; workspaces with anything in them."""
    x, u, g = logits(B, V, F32, 7)
    args = dict(logits=x, u=col(u), temperature=torch.full((B,), 0.8, device="cuda"), top_k=torch.full((B,), 50, dtype=I32, device="cuda"),
                top_p=torch.full((B,), 0.9, device="cuda"), min_p=torch.zeros(B, device="cuda"))
    ws = torch.full((max(16, ta.sample_workspace_bytes(B, V)),), 0xFF, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = ta.sample_logits(**args, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        token, logp = ta.sample_logits(**args)
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = ta.sample_logits(**args)
        assert torch.equal(token, want[0]) and torch.equal(logp, want[1])
        x.copy_(torch.randn(B, V, generator=g).cuda() * (i + 1))
        args["u"].copy_(torch.rand(B, generator=g).cuda())
        args["top_k"].fill_([0, 5, 3000, 0][i]), args["temperature"].fill_([1.0, 0.0, 0.5, 1.0][i])
