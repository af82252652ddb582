"""Long sums of the serving calls on whole numbers, so that fp32 makes no error in them and a
block of keys or a step of K that is left out, doubled or read elsewhere shows, which a bound
for the roundings of a million terms would hide.

Attention: scores are 0, -1, -2 or -3 with a scale whose product with log2(e) is 1 in fp32
(fp32's ln 2), so that weights are powers of two; values are whole numbers up to 8.  Both
sums are multiples of 2^-3 below 2^21: exact in any order.  What is left is the exponential
(2^-23, were it not exact for whole numbers), once more where parts and waves meet, the
quotient (two roundings of 2^-24), and fp32's ln 2 in the scale (3 2^-28): 2^-21 of the
weighted sizes together; for LSE the logarithm's ulp and its product's (2^-22 of it) besides.

Products: A and B hold -2 .. 2, sums stay below 4 (2^22 - 8) < 2^24."""

import pytest

torch = pytest.importorskip("torch")

from paper_2504_17577_amd import tileattn as ta  # noqa: E402

BF16, F32, E4M3, I32 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.int32
LN2 = 0.693147182464599609375   # in fp32


def numbers(g, *shape, D, dev):
    s = -torch.randint(0, 4, shape, generator=g, device=dev)
    v = torch.randint(-8, 9, shape + (D,), generator=g, device=dev)
    return s, v


def exact(s, v):
    """O, LSE and the weighted mean of |v| for one row of scores s [n] and values v [n, D]."""
    p = torch.exp2(s.double())
    return p @ v.double() / p.sum(), p.sum().log(), p @ v.double().abs() / p.sum()


def test_a_lost_block_would_show():
    """Without any one of the 16-key blocks, O or LSE is further off than the tolerance."""
    n, D = 200000, 64
    s, v = numbers(torch.Generator().manual_seed(0), n, D=D, dev="cpu")
    o, lse, size = exact(s, v)
    p = torch.exp2(s.double())
    pb, vb = p.view(-1, 16).sum(1), (p[:, None] * v.double()).view(-1, 16, D).sum(1)
    for sign in (-1, 1):                     # left out, or twice
        o2 = (p @ v.double() + sign * vb) / (p.sum() + sign * pb)[:, None]
        assert (((o2 - o).abs() / (2.0 ** -21 * size)).amax(1) > 10).all()
        assert (((p.sum() + sign * pb).log() - lse).abs() > 3 * (2.0 ** -21 + 2.0 ** -22 * lse)).all()


CASES = [
    # (lens, query heads to a K/V head, Hkv, D, page, parts)
    ([200000, 131073], 8, 1, 64, 1 << 17, (None, 0, 3)),
    ([60000], 2, 8, 128, 64, (None, 4096, 1)),
    ([100001], 4, 2, 128, 64, (None, 511)),
    ([8191, 8192, 8193, 4095, 64, 63, 65, 0, 1], 20, 2, 64, 16, (None, 0, 100)),
    ([7 * i % 330 for i in range(700)], 4, 2, 128, 16, (None, 0, 512, 4096)),
    ([64, 1, 63, 64, 0, 49], 3, 2, 64, 16, (None, 0, 1, 5)),       # as long as the table has room for
    ([2048, 2048], 33, 1, 128, 1024, (None, 0, 2)),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, E4M3], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("case", CASES, ids=[f"{len(c[0])}x{max(c[0])}-g{c[1]}-d{c[3]}" for c in CASES])
def test_every_key_counts_once(case, dtype):
    lens, group, Hkv, D, P, all_parts = case
    g = torch.Generator(device="cuda").manual_seed(len(lens) + D)
    need = [-(-n // P) for n in lens]
    order = torch.randperm(sum(need) + 2, generator=g, device="cuda").to(I32)
    table = torch.full((len(lens), max(need)), -1, dtype=I32, device="cuda")
    kc, vc = (torch.full((sum(need) + 2, Hkv, P, D), float("nan"), device="cuda").to(dtype) for _ in range(2))
    want = []
    for b, n in enumerate(lens):
        pages, order = order[:need[b]], order[need[b]:]
        table[b, :need[b]] = pages
        want.append([])
        if n == 0:
            continue
        s, v = numbers(g, Hkv, n, D=D, dev="cuda")
        for h in range(Hkv):
            want[b].append(exact(s[h], v[h]))
            k = torch.full((need[b] * P, D), float("nan"), device="cuda")
            k[:n] = torch.randint(-8, 9, (n, D), generator=g, device="cuda").float()
            k[:n, 7] = s[h].float()
            # (an 8-bit tensor is filled through its bytes)
            kc.view(torch.uint8)[pages.long(), h] = k.view(need[b], P, D).to(dtype).view(torch.uint8)
            k[:n] = v[h].float()
            vc.view(torch.uint8)[pages.long(), h] = k.view(need[b], P, D).to(dtype).view(torch.uint8)
    q = torch.zeros(len(lens), Hkv * group, D, dtype=BF16, device="cuda")
    q[:, :, 7] = 1
    lens_t = torch.tensor(lens, dtype=I32, device="cuda")
    for parts in all_parts:
        print(f"  parts {parts}", flush=True)
        o, lse = ta.attn_decode_paged(q, kc, vc, table, lens_t, scale=LN2, num_parts=parts)
        o, lse = o.double().view(-1, Hkv, group, D), lse.double().view(-1, Hkv, group)
        for b, n in enumerate(lens):
            if n == 0:
                assert (o[b] == 0).all() and torch.isneginf(lse[b]).all()
            for h, (wo, wl, size) in enumerate(want[b]):
                assert ((o[b, h] - wo).abs() <= 2.0 ** -21 * size + 1e-30).all(), (b, h)
                assert ((lse[b, h] - wl).abs() <= 2.0 ** -21 + 2.0 ** -22 * wl.abs()).all(), (b, h)


@pytest.mark.gpu
@pytest.mark.parametrize("splits", [None, 1, 7, 64])
@pytest.mark.parametrize("M,N,K", [
    (1, 8, (1 << 22) - 8), (64, 8, (1 << 22) - 8), (70, 8, (1 << 22) - 8), (300, 264, 400008), (9, 4104, 100008),
])
def test_every_step_of_a_long_product_counts_once(M, N, K, splits):
    g = torch.Generator(device="cuda").manual_seed(M)
    a, b = (torch.randint(-2, 3, s, generator=g, device="cuda").to(BF16) for s in ((M, K), (K, N)))
    want = torch.zeros(M, N, dtype=torch.float64, device="cuda")
    for k in range(0, K, 1 << 18):
        want += a[:, k:k + (1 << 18)].double() @ b[k:k + (1 << 18)].double()
    got = ta.gemm_bf16_epilogue(a, b, num_splits=splits)
    assert torch.equal(got.double(), want)
