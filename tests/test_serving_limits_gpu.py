"""The serving calls at the sizes where an index could go wrong: operands past 2^31
elements and 4 GiB, the largest row counts and divisions, many sequences, very
large pages, one scale without the other, two tokens for one place."""
import numpy as np
import pytest

from oracle import serving

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, F32, E4M3, I32 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.int32


@pytest.fixture(scope="module")
def ta():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2504_17577_amd import tileattn
    tileattn.lib()
    return tileattn


@pytest.mark.parametrize("M,N,K,out", [
    (1 << 20, 8, 2056, BF16),        # the most rows; A of 4.3 GB
    (3, 600000, 4096, F32),          # B of 4.9 GB, few rows
    (70, 600000, 4096, BF16),        # the same through the tiled kernel
    (70000, 40000, 72, F32),         # C of 11 GB
    (1, 8, (1 << 22) - 8, F32),      # the longest K
    (64, (1 << 24) - 8, 8, BF16),    # the widest N
])
def test_large_products(ta, M, N, K, out):
    g = torch.Generator(device="cuda").manual_seed(1)
    draw = lambda *s: torch.empty(s, dtype=BF16, device="cuda").normal_(generator=g)   # noqa: E731
    a, b, bias = draw(M, K), draw(K, N), draw(N)
    c = ta.gemm_bf16_epilogue(a, b, bias=bias, activation="relu", out_dtype=out)
    rows = sorted({0, M // 3, M - 1, max(0, M - 129)})
    cols = torch.tensor(sorted({0, 5 % N, N // 2, max(0, N - 130), N - 1}), device="cuda")
    sel = b[:, cols].double()
    for m in rows:
        want = (a[m].double() @ sel + bias[cols].double()).clamp(min=0)
        size = a[m].double().abs() @ sel.abs() + bias[cols].double().abs()
        # K + 2 roundings of 2^-24 of the sum of sizes, and half a step of the result's type
        tol = (K + 2) * 2.0 ** -24 * size + torch.finfo(out).eps / 2 * want + 1e-30
        assert ((c[m, cols].double() - want).abs() <= tol).all(), m
    part = torch.isfinite(c[rows])
    assert part.all()


@pytest.mark.parametrize("splits", [1, 64])
@pytest.mark.parametrize("M", [64, 65])
def test_products_at_the_kernels_border(ta, M, splits):
    g = torch.Generator(device="cuda").manual_seed(M)
    a = torch.randn(M, 2056, generator=g, device="cuda").to(BF16)
    b = torch.randn(2056, 392, generator=g, device="cuda").to(BF16)
    want = a.double() @ b.double()
    tol = 2058 * 2.0 ** -24 * (a.double().abs() @ b.double().abs())
    assert ((ta.gemm_bf16_epilogue(a, b, num_splits=splits).double() - want).abs() <= tol).all()


def plain(q, kc, vc, table, lens, scale, ks=None, vs=None):
    """float64 on the GPU, sequence by sequence."""
    B, Hq, D = q.shape
    Hkv, P = kc.shape[1], kc.shape[2]
    o = torch.zeros(B, Hq, D, dtype=torch.float64, device=q.device)
    lse = torch.full((B, Hq), -np.inf, dtype=torch.float64, device=q.device)
    for b, n in enumerate(lens.tolist()):
        if n == 0:
            continue
        pages = table[b, :-(-n // P)].long()
        k, v = ((c.view(torch.uint8)[pages].view(c.dtype) if c.dtype == E4M3 else c[pages]).double().transpose(0, 1)
                .reshape(Hkv, -1, D)[:, :n] for c in (kc, vc))
        k = k if ks is None else k * ks.double()[:, None, None]
        v = v if vs is None else v * vs.double()[:, None, None]
        s = scale * (q[b].double().view(Hkv, Hq // Hkv, D) @ k.transpose(1, 2).contiguous())
        lse[b] = torch.logsumexp(s, 2).view(Hq)
        o[b] = (torch.softmax(s, 2) @ v).view(Hq, D)
    return o, lse


def agree(got, want, D):
    """fp32 arithmetic on products of unit normals: scores of at most 9 in size summed
    of D terms (2 (D + 4) 2^-24 of the sum of sizes, below 1.5 D^0.5), exponentials to
    2^-21, sums over the keys to 2^-18 at most here, for |V| up to 6."""
    tol = 6 * (2 * (D + 4) * 2.0 ** -24 * 1.5 * D ** 0.5 + 2.0 ** -21 + 2.0 ** -18)
    o, lse = got[0].double(), got[1].double()
    assert torch.equal(torch.isinf(lse), torch.isinf(want[1]))
    fin = torch.isfinite(lse)
    assert ((o - want[0]).abs() <= tol).all() and ((lse - want[1])[fin].abs() <= tol).all()


@pytest.mark.parametrize("B,Hq,Hkv,D,P,top,parts", [
    (3000, 4, 2, 64, 16, 40, None), (3000, 4, 2, 64, 16, 40, 512), (500, 1, 1, 128, 16, 300, 4096),
    (2, 8, 1, 64, 1 << 17, 200000, None), (1, 16, 8, 128, 64, 60000, 4096), (5, 256, 4, 128, 32, 500, 7),
])
def test_batches_at_their_largest(ta, B, Hq, Hkv, D, P, top, parts):
    g = torch.Generator(device="cuda").manual_seed(B)
    per = -(-top // P)
    kc, vc = (torch.empty(B * per, Hkv, P, D, dtype=BF16, device="cuda").normal_(generator=g) for _ in range(2))
    table = torch.randperm(B * per, generator=g, device="cuda").to(I32).view(B, per)
    lens = torch.randint(0, top + 1, (B,), generator=g, device="cuda").to(I32)
    lens[0] = top
    q = torch.empty(B, Hq, D, dtype=BF16, device="cuda").normal_(generator=g)
    got = ta.attn_decode_paged(q, kc, vc, table, lens, num_parts=parts)
    agree(got, plain(q, kc, vc, table, lens, D ** -0.5), D)


@pytest.mark.parametrize("which", ["k", "v"])
def test_one_scale_without_the_other(ta, which):
    g = torch.Generator(device="cuda").manual_seed(4)
    kc, vc = (torch.randn(12, 2, 16, 64, generator=g, device="cuda").to(E4M3) for _ in range(2))
    table = torch.randperm(12, generator=g, device="cuda").to(I32).view(3, 4)
    lens = torch.tensor([64, 1, 33], dtype=I32, device="cuda")
    q = torch.randn(3, 4, 64, generator=g, device="cuda").to(BF16)
    sc = torch.tensor([0.5, 0.9], device="cuda")
    ks, vs = (sc, None) if which == "k" else (None, sc)
    got = ta.attn_decode_paged(q, kc, vc, table, lens, k_scale=ks, v_scale=vs)
    agree(got, plain(q, kc, vc, table, lens, 0.125, ks, vs), 64)
    new = torch.randn(3, 2, 64, generator=g, device="cuda").to(BF16)
    ta.kv_cache_append(new, new, kc, vc, table, lens - 1, k_scale=ks, v_scale=vs)
    for c, s in ((kc, ks), (vc, vs)):
        for b in range(3):
            t = int(lens[b]) - 1
            x = new[b].float() if s is None else new[b].float() / s[:, None]
            want = x.clamp(-448, 448).to(E4M3)
            assert torch.equal(c[table[b, t // 16].long(), :, t % 16].view(torch.uint8), want.view(torch.uint8))


@pytest.mark.parametrize("parts", [0, 7])
@pytest.mark.parametrize("n", [1, 16, 300])
def test_every_score_minus_infinity(ta, n, parts):
    """The weights are 0 / 0: NaN, not the zeros of an idle slot."""
    D, P = 64, 16
    per = -(-n // P)
    g = torch.Generator(device="cuda").manual_seed(n)
    kc, vc = (torch.randn(2 * per, 1, P, D, generator=g, device="cuda").to(BF16) for _ in range(2))
    table = torch.arange(2 * per, dtype=I32, device="cuda").view(2, per)
    lens = torch.tensor([n, 0], dtype=I32, device="cuda")
    kc[:, :, :, 5] = float("-inf")
    q = torch.rand(2, 3, D, generator=g, device="cuda").add(0.5).to(BF16)
    o, lse = ta.attn_decode_paged(q, kc, vc, table, lens, num_parts=parts)
    assert torch.isnan(o[0]).all() and torch.isneginf(lse[0]).all()
    assert (o[1] == 0).all() and torch.isneginf(lse[1]).all()
    want = plain(q[:1], kc, vc, table, lens[:1], 0.125)
    assert torch.isnan(want[0]).all() and torch.isneginf(want[1]).all()


def test_two_tokens_for_one_place(ta):
    """Which of them it holds is not defined; that it holds one of them, piece by piece,
    and that nothing else is touched, is."""
    kc, vc = (torch.zeros(4, 2, 16, 128, dtype=BF16, device="cuda") for _ in range(2))
    new = torch.stack([torch.full((2, 128), 1.0), torch.full((2, 128), 2.0), torch.full((2, 128), 3.0)]).to(BF16).cuda()
    table = torch.arange(4, dtype=I32, device="cuda").view(2, 2)
    seq = torch.tensor([1, 1, 0], dtype=I32, device="cuda")
    ta.kv_cache_append(new, -new, kc, vc, table, torch.tensor([17, 17, 3], dtype=I32, device="cuda"), seq=seq)
    for c, sign in ((kc, 1), (vc, -1)):
        got = (sign * c[3, :, 1].float()).view(2, 16, 8)
        assert ((got == 1) | (got == 2)).all() and (got == got[:, :, :1]).all()
        assert (sign * c[0, :, 3] == 3).all()
        c[3, :, 1] = 0
        c[0, :, 3] = 0
        assert (c == 0).all()


def test_append_past_4_gib(ta):
    P, D = 1024, 128
    pages = (1 << 32) // (P * D * 2) + 8
    kc, vc = (torch.zeros(pages, 1, P, D, dtype=BF16, device="cuda") for _ in range(2))
    table = torch.tensor([[pages - 1, 3, pages // 2 + 1]], dtype=I32, device="cuda")
    pos = torch.tensor([5, P + 6, 2 * P + 7, P - 1], dtype=I32, device="cuda")
    new = torch.arange(1, 5, device="cuda").to(BF16).view(4, 1, 1).expand(4, 1, D).contiguous()
    ta.kv_cache_append(new, new, kc, vc, table, pos, seq=torch.zeros(4, dtype=I32, device="cuda"))
    for c in (kc, vc):
        for i, (page, row) in enumerate([(pages - 1, 5), (3, 6), (pages // 2 + 1, 7), (pages - 1, P - 1)]):
            assert (c[page, 0, row] == i + 1).all()
        assert int((c != 0).sum()) == 4 * D


def test_oracle_and_plain_agree(ta):
    """(the GPU reference of this file against the oracle that the other tests use)"""
    g = torch.Generator(device="cuda").manual_seed(9)
    kc, vc = (torch.randn(6, 2, 16, 64, generator=g, device="cuda").to(BF16) for _ in range(2))
    table = torch.randperm(6, generator=g, device="cuda").to(I32).view(2, 3)
    lens, q = torch.tensor([40, 0], dtype=I32, device="cuda"), torch.randn(2, 4, 64, generator=g, device="cuda").to(BF16)
    f = lambda t: t.double().cpu().numpy()   # noqa: E731
    want = serving.attn_paged(f(q), f(kc), f(vc), table.cpu().numpy(), lens.tolist(), 0.125)
    o, lse = plain(q, kc, vc, table, lens, 0.125)
    np.testing.assert_allclose(f(o), want[0], atol=1e-12)
    np.testing.assert_allclose(f(lse), want[1], atol=1e-12)
