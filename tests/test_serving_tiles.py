"""gemm_bf16_epilogue by the tiles it runs in: all columns in 256 x 256 tiles, the first of
them and the others in 128 x 128 tiles with and without a split of K, 128 x 128 tiles alone,
each with ragged sizes, both result types and every epilogue.  Each shape's kernels are
asserted on the CPU, so that another choice cannot leave a path without its test.

Matrices hold small whole numbers (B's and the residual's as multiples of 2^-7), so that
every sum is exact in fp32 (below 2^24 units): results without an activation are equal to
the exact ones, rounded once, and anything left out, doubled or misplaced shows."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2504_17577_amd import tileattn as ta  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
UNIT = 2.0 ** -7

TILES = [
    # (M, N, K, num_splits, ranges of K, columns in 256 x 256 tiles)
    (4096, 8192, 1024, None, 1, 8192),
    (4090, 8184, 4104, None, 1, 8184),     # all columns, ragged on every side
    (4090, 8184, 1032, 3, 3, 8184),        # (nothing is left to split)
    (1500, 14344, 4104, None, 1, 10752),   # two kinds of tiles, K whole
    (2100, 8400, 1032, None, 1, 7168),
    (4000, 8200, 4104, None, 13, 8192),    # two kinds, K split in the second
    (1500, 14344, 4104, 3, 3, 10752),
    (2000, 2056, 200, None, 1, 0),         # 128 x 128, more than one a CU
    (2000, 2056, 8, None, 1, 0),
    (300, 264, 1032, 1, 1, 0),             # 128 x 128, few
    (300, 264, 1032, 5, 5, 0),
]
IDS = [f"{m}x{n}x{k}-{s}" for m, n, k, s, _, _ in TILES]


@pytest.mark.parametrize("case", TILES, ids=IDS)
def test_shapes_take_their_tiles(case):
    M, N, K, splits, ranges, large = case
    used = ta.gemm_epilogue_plan(M, N, K) if splits is None else splits
    assert used == ranges and ta.gemm_epilogue_route(M, N, K, used) == large


def test_route_of_all_sizes():
    for M in (1, 64, 65, 256, 1000, 4096, 100000):
        for N in (8, 256, 4096, 65536):
            for K in (8, 64, 1000, 8192):
                for sp in (1, 2, 64):
                    n = ta.gemm_epilogue_route(M, N, K, sp)
                    assert 0 <= n <= N and (n == N or n % 256 == 0) and (M > 64 or n == 0)
    for bad, status in [((0, 8, 8, 1), 2), ((1, 8, -8, 1), 2), ((1, 8, 8, 0), 2), ((1, 8, 8, 65), 2), ((1, 12, 8, 1), 3)]:
        with pytest.raises(ta.TileAttnError) as e:
            ta.gemm_epilogue_route(*bad)
        assert e.value.status == status
    assert ta.lib().gemm_epilogue_route(1, 8, 8, 1, None) == 1


def operands(M, N, K):
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    draw = lambda top, *s: torch.randint(-top, top + 1, s, generator=g, device="cuda").to(BF16)   # noqa: E731
    return draw(3, M, K), draw(3, K, N) * UNIT, draw(255, N) * UNIT, draw(255, M, N) * UNIT


def activated(x, act):
    """The activation in 64 bits, and what an fp32 evaluation may be off by, of its value."""
    if act == "relu":
        return x.clamp(min=0), 0.0
    if act == "gelu":
        # erfc's argument z = x / sqrt 2 is off by 1.3 2^-24 of itself (the product half an ulp, the
        # constant 2^-25.8), and erfc(z), whose slope is below 2 (z + 1 / z) erfc(z) for z > 0 and
        # below 2 erfc(z) for others, by (2 z^2 + 2) times that
        return 0.5 * x * torch.erfc(-x / math.sqrt(2)), 2.0 ** -20 + (x * x + 2) * 1.3 * 2.0 ** -24
    u = x if act == "silu" else 2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)
    # the sigmoid 2^-21 and as much in its exponent's last bits; the tanh gelu's u 7 2^-24 of
    # itself; a bf16 C's sigmoid 2^-21 + 1.25 2^-24 of |u|
    return x * torch.sigmoid(u), 2.0 ** -20 + (1.25 + 7 * (act == "gelu_tanh")) * 2.0 ** -24 * u.abs()


def check_product(M, N, K, splits, dt):
    a, b, bias, res = operands(M, N, K)
    x = a.double() @ b.double()
    print(f"  {M} x {N} x {K} splits {splits}", flush=True)
    for act, has_bias, has_res in [("none", 0, 0), ("none", 1, 1), ("relu", 1, 1), ("silu", 1, 0), ("gelu", 0, 1), ("gelu_tanh", 1, 0)]:
        r = res.to(dt) if has_res else None
        got = ta.gemm_bf16_epilogue(a, b, bias=bias if has_bias else None, activation=act, residual=r, out_dtype=dt,
                                    num_splits=splits)
        y = x + bias.double() if has_bias else x
        of = 0.0
        if act != "none":
            y, of = activated(y, act)
        want = y + res.double() if has_res else y
        if act in ("none", "relu"):
            same = got == want.float().to(dt)
            assert same.all(), f"{act}: {int((~same).sum())} of {same.numel()} differ, first {(~same).nonzero()[0].tolist()}"
        else:
            # of the activation, the sum with the residual, half a step of bf16
            tol = of * y.abs() + (2.0 ** -24 + (dt == BF16) * 2.0 ** -8) * want.abs() + 2.0 ** -119
            err = (got.double() - want).abs()
            assert (err <= tol).all(), f"{act}: {float((err / tol).max()):.2f} of the tolerance"


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("case", TILES, ids=IDS)
def test_product_in_its_tiles(case, dt):
    check_product(*case[:4], dt)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16], ids=["fp32", "bf16"])
def test_large_tiles_in_place(dt):
    a, b, _, res = operands(4090, 8184, 72)
    assert ta.gemm_epilogue_route(4090, 8184, 72, 2) == 8184
    want = (a.double() @ b.double() + res.double()).float().to(dt)
    c = res.to(dt)
    assert ta.gemm_bf16_epilogue(a, b, residual=c, out=c, out_dtype=dt, num_splits=2) is c
    assert torch.equal(c, want)
