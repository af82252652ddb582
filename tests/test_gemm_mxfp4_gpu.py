"""GPU parity of gemm_mxfp4_epilogue against the float64 oracle on the numbers that the
codes stand for; tolerances are the oracle's bounds for fp32 sums of exact products,
plus half a step (2^-8 of the value) for a bf16 result."""
import numpy as np
import pytest

from oracle import more_serving as ms
from oracle import serving

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, F32, U8 = torch.bfloat16, torch.float32, torch.uint8


@pytest.fixture(scope="module")
def ta():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2504_17577_amd import tileattn
    tileattn.lib()
    return tileattn


def f64(t):
    return t.double().cpu().numpy()


def weights(N, K, g, spread=1):
    """Random codes and scales around K^-1/2, and their numbers."""
    w = torch.randint(0, 256, (N, K // 2), generator=g, dtype=U8)
    e = 125 - int(np.log2(K)) // 2
    s = torch.randint(e - spread, e + spread + 1, (N, K // 32), generator=g, dtype=U8)
    return w.cuda(), s.cuda(), ms.mx_values(w.numpy(), s.numpy())


SIZES = [
    # (M, N, K): few rows in blocks of 16, strips of 16, 32 and 64 columns, K in parts of steps
    (1, 8, 32), (1, 4096, 4096), (1, 72, 992), (2, 64, 64), (5, 136, 288), (16, 128, 512), (17, 1000, 1056),
    (24, 2048, 1024), (32, 256, 4096), (33, 520, 96), (48, 4096, 256), (64, 136, 2080), (49, 8, 3200),
    (3, 8200, 160), (9, 6152, 640), (16, 12296, 2080), (7, 10248, 2176), (40, 8208, 224), (64, 16400, 128), (20, 20008, 96), (64, 17000, 416),
    # tiles: one row over, one short, columns and K in parts
    (65, 200, 544), (96, 1024, 1024), (127, 136, 128), (128, 128, 64), (129, 264, 352), (200, 1000, 992),
    (256, 256, 256), (300, 8, 32), (389, 520, 1056), (513, 1032, 224), (130, 2056, 3200),
]
EPILOGUE = [("none", 0, 0), ("relu", 1, 0), ("gelu", 1, 1), ("gelu_tanh", 0, 1), ("silu", 1, 1), ("none", 1, 1)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_against_oracle(ta, M, N, K):
    g = torch.Generator().manual_seed(M + N + K)
    a = torch.randn(M, K, generator=g).to(BF16).cuda()
    w, s, v = weights(N, K, g)
    bias, res = torch.randn(N, generator=g).to(BF16).cuda(), torch.randn(M, N, generator=g).cuda()
    for i, (act, has_bias, has_res) in enumerate(EPILOGUE):
        dt = F32 if i % 2 == (M % 2) else BF16
        r = res.to(dt) if has_res else None
        c, tol = serving.gemm_epilogue(f64(a), v.T, f64(bias) if has_bias else None, act, f64(r) if has_res else None)
        if dt == BF16:
            tol = tol + 2.0 ** -8 * np.abs(c)
        for parts in (None, 0, 1, 3, 37, 256):
            got = ta.gemm_mxfp4_epilogue(a, w, s, bias=bias if has_bias else None, activation=act, residual=r, out_dtype=dt,
                                         num_parts=parts)
            assert got.dtype == dt and got.shape == (M, N)
            err = np.abs(f64(got) - c)
            print(f"  {act} {has_bias} {has_res} {dt} parts {parts}: of bound {(err / tol).max():.2f}", flush=True)
            assert (err <= tol).all()


@pytest.mark.parametrize("M,N,K", [(1, 264, 1056), (17, 520, 4128), (64, 72, 288), (100, 264, 1056), (300, 520, 416)])
def test_every_weight_counts_once(ta, M, N, K):
    """Sums of small whole numbers, exact in fp32 (below 2^24): a lost, doubled or
    misplaced code, scale or step shows as another number."""
    g = torch.Generator().manual_seed(K)
    a = torch.randint(-3, 4, (M, K), generator=g).to(BF16).cuda()
    w = torch.randint(0, 256, (N, K // 2), generator=g, dtype=U8)
    s = torch.randint(128, 131, (N, K // 32), generator=g, dtype=U8)
    want = f64(a) @ ms.mx_values(w.numpy(), s.numpy()).T
    for parts in (None, 1, 3):
        got = ta.gemm_mxfp4_epilogue(a, w.cuda(), s.cuda(), num_parts=parts)
        np.testing.assert_array_equal(f64(got), want)


@pytest.mark.parametrize("M", [1, 40, 300])
def test_one_weight_at_a_time(ta, M):
    """A unit row of A picks one column of W: every code, scales from end to end (subnormal
    results left out), each in its own place."""
    N, K = 512, 256
    g = torch.Generator().manual_seed(M)
    w = torch.randint(0, 256, (N, K // 2), generator=g, dtype=U8)
    s = torch.randint(3, 250, (N, K // 32), generator=g, dtype=U8)
    v = ms.mx_values(w.numpy(), s.numpy())
    for k0 in (0, 31, 37, 200):
        a = torch.zeros(M, K, dtype=BF16)
        cols = (k0 + np.arange(M) * 5) % K
        a[torch.arange(M), torch.from_numpy(cols)] = 1
        got = ta.gemm_mxfp4_epilogue(a.cuda(), w.cuda(), s.cuda())
        np.testing.assert_array_equal(f64(got), v[:, cols].T)


@pytest.mark.parametrize("M,N,K", [(300, 12296, 1056), (1021, 4232, 8224), (700, 8200, 2080), (65, 20000, 96)])
def test_large_tiles(ta, M, N, K):
    """Sizes at which tiles of 256 columns are chosen, and others; the oracle's arithmetic on
    the GPU (float64)."""
    g = torch.Generator().manual_seed(N)
    a, (w, s, v) = torch.randn(M, K, generator=g).to(BF16).cuda(), weights(N, K, g)
    bias, r = torch.randn(N, generator=g).to(BF16).cuda(), torch.randn(M, N, generator=g).to(BF16).cuda()
    v = torch.from_numpy(v.T.copy()).cuda()
    x = a.double() @ v + bias.double()
    size = a.double().abs() @ v.abs() + bias.double().abs()
    y = x * torch.sigmoid(x)
    # as oracle.serving.gemm_epilogue's, and half a step of bf16
    tol = 1.13 * (K + 2) * 2.0 ** -24 * size + 2.0 ** -20 * y.abs() + (2.0 ** -24 + 2.0 ** -8) * (y + r.double()).abs() + 1e-30
    for parts in (None, 0, 37, 256, 512):
        got = ta.gemm_mxfp4_epilogue(a, w, s, bias=bias, activation="silu", residual=r, out_dtype=BF16, num_parts=parts)
        err = (got.double() - y - r.double()).abs()
        print(f"  parts {parts}: of bound {float((err / tol).max()):.2f}", flush=True)
        assert (err <= tol).all()


@pytest.mark.parametrize("M", [5, 24, 60])
def test_scales_at_any_address(ta, M):
    """K in whole steps, the scales at each byte of a dword."""
    N, K = 10304, 2304
    g = torch.Generator().manual_seed(M)
    a, (w, s, _) = torch.randn(M, K, generator=g).to(BF16).cuda(), weights(N, K, g)
    want = ta.gemm_mxfp4_epilogue(a, w, s)
    room = torch.zeros(N * K // 32 + 8, dtype=U8, device="cuda")
    for at in range(1, 4):
        t = room[at:at + N * K // 32].view(N, K // 32)
        t.copy_(s)
        assert torch.equal(ta.gemm_mxfp4_epilogue(a, w, t), want)


@pytest.mark.parametrize("M", [1, 40, 300])
@pytest.mark.parametrize("dt", [F32, BF16], ids=["fp32", "bf16"])
def test_onto_the_residual_in_place(ta, M, dt):
    g = torch.Generator().manual_seed(M)
    a, (w, s, _) = torch.randn(M, 1056, generator=g).to(BF16).cuda(), weights(264, 1056, g)
    x = torch.randn(M, 264, generator=g).to(dt).cuda()
    for parts in (1, 3):
        y = x.clone()
        want = ta.gemm_mxfp4_epilogue(a, w, s, residual=x, out_dtype=dt, num_parts=parts)
        assert ta.gemm_mxfp4_epilogue(a, w, s, residual=y, out=y, out_dtype=dt, num_parts=parts) is y
        assert torch.equal(y, want)


@pytest.mark.parametrize("M", [1, 20, 100, 300])
def test_infinities_and_nan(ta, M):
    """What a row of A or W holds stays in that row or column of C, in a last part of a
    step too; a scale of 255 is NaN."""
    K = 160
    a = torch.ones(M, K, dtype=BF16, device="cuda")
    w = torch.full((200, K // 2), 0x22, dtype=U8, device="cuda")     # ones
    s = torch.full((200, K // 32), 127, dtype=U8, device="cuda")
    a[M - 1, K - 1], s[199, K // 32 - 1], s[7, 0] = float("inf"), 255, 255
    w[3, K // 2 - 1] = 0xA2                                          # its last number -1
    c = ta.gemm_mxfp4_epilogue(a, w, s)
    want = torch.full((M, 200), float(K))
    want[:, 3] = K - 2
    want[M - 1] = float("inf")
    want[M - 1, 3] = float("-inf")
    want[:, 199], want[:, 7] = float("nan"), float("nan")
    np.testing.assert_array_equal(c.cpu().numpy(), want.numpy())


@pytest.mark.parametrize("M", [3, 100])
def test_guarded_rows(ta, M):
    """Nothing beside C is written, nothing beside A, W and the scales is read (NaN and
    255 stand there)."""
    N, K = 136, 288
    g = torch.Generator().manual_seed(M)
    a, (w, s, v) = torch.randn(M, K, generator=g).to(BF16).cuda(), weights(N, K, g)
    big = torch.full((M * K + 4096,), float("nan"), dtype=BF16, device="cuda")
    ws = torch.full((N * K // 2 + 4096,), 0x77, dtype=U8, device="cuda")
    ss = torch.full((N * K // 32 + 4096 + 1,), 255, dtype=U8, device="cuda")
    a2, w2 = big[2048:2048 + M * K].view(M, K), ws[2048:2048 + N * K // 2].view(N, K // 2)
    s2 = ss[2049:2049 + N * K // 32].view(N, K // 32)                # an odd address
    a2.copy_(a), w2.copy_(w), s2.copy_(s)
    out = torch.full((M * N + 4096,), 5.0, device="cuda")
    c = out[2048:2048 + M * N].view(M, N)
    for parts in (1, 2):
        ta.gemm_mxfp4_epilogue(a2, w2, s2, out=c, num_parts=parts)
        want, tol = serving.gemm_epilogue(f64(a), v.T)
        assert (np.abs(f64(c) - want) <= tol).all()
        assert (out[:2048] == 5).all() and (out[2048 + M * N:] == 5).all()


def test_rows_past_4_gib(ta):
    """Codes whose byte offset passes 2^32: the last strip and tile."""
    N, K = 1 << 16, 1 << 18
    w = torch.zeros(N, K // 2, dtype=U8, device="cuda")
    s = torch.full((N, K // 32), 127, dtype=U8, device="cuda")
    w[N - 1, K // 2 - 1], w[N // 2, 5] = 0x40, 0x03
    for M in (2, 65):
        a = torch.ones(M, K, dtype=BF16, device="cuda")
        c = ta.gemm_mxfp4_epilogue(a, w, s)
        assert (c[:, N - 1] == 2).all() and (c[:, N // 2] == 1.5).all() and int((c != 0).sum()) == 2 * M
