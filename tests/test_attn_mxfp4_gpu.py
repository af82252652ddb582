"""GPU parity of attention over a paged cache held in 4 bits (attn_decode_paged on
uint8 caches) against the float64 oracle on the numbers that the codes stand for.
Tolerances and bounds are those of the other cache types (test_serving_gpu); a place
that no sequence holds has a scale of 255 (NaN), and unused entries of the table point
outside, so that anything read past a sequence's end shows."""
import numpy as np
import pytest

from oracle import more_serving as ms
from oracle import serving
from test_serving_gpu import ATTN, BF16, F32, Cache, check, f64

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U8 = torch.uint8


@pytest.fixture(scope="module")
def ta():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2504_17577_amd import tileattn
    tileattn.lib()
    return tileattn


class Cache4(Cache):
    """Cache's layout in 4 bits; k and v are the numbers, in float32."""

    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        self.codes, self.scales4 = [], []
        for x in (self.k, self.v):
            codes, scales = ms.mx_pack(x.float().cpu().numpy())
            nan = np.isnan(x.float().cpu().numpy()).any(-1)
            codes[nan] = np.random.default_rng(0).integers(0, 256, codes[nan].shape)
            self.codes.append(torch.from_numpy(codes).cuda())
            self.scales4.append(torch.from_numpy(scales).cuda())
        self.k, self.v = (torch.from_numpy(ms.mx_values(c.cpu().numpy(), s.cpu().numpy())).float().cuda()
                          for c, s in zip(self.codes, self.scales4))

    def args(self):
        return *self.codes, self.table, self.lens

    def scales(self):
        return dict(k_scale=self.scales4[0], v_scale=self.scales4[1])


def reference(q, c, scale):
    return serving.attn_paged(f64(q), f64(c.k), f64(c.v), c.table.cpu().numpy(), c.lens.tolist(), scale)


CASES = [c[:5] for c in ATTN if not c[5]] + [
    ([1, 0, 37], 4, 2, 64, 16), ([1500, 64, 63], 16, 1, 128, 64), ([513, 2], 40, 2, 64, 128), ([9001], 8, 2, 128, 64),
    ([9001], 8, 2, 64, 16), ([3000, 2999], 32, 1, 128, 16),
]


@pytest.mark.parametrize("case", CASES, ids=[f"{len(c[0])}x{max(c[0])}-h{c[1]}.{c[2]}-d{c[3]}-p{c[4]}" for c in CASES])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
def test_against_oracle(ta, case, dtype):
    lens, Hq, Hkv, D, P = case
    c = Cache4(lens, Hkv, D, P, seed=len(lens))
    q = torch.randn(len(lens), Hq + 3, D, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()[:, 1:Hq + 1]
    o = torch.full((len(lens), Hq, D), float("nan"), dtype=dtype, device="cuda")
    lse = torch.full((len(lens), Hq), float("nan"), device="cuda")
    ref = reference(q, c, D ** -0.5)
    for parts in (None, 0, 1, 3, 37, 512):
        print(f"  parts {parts}", flush=True)
        o.fill_(float("nan")), lse.fill_(float("nan"))
        r = ta.attn_decode_paged(q, *c.args(), **c.scales(), out=o, lse=lse, num_parts=parts, out_dtype=dtype)
        assert r[0] is o and r[1] is lse
        check(c, o, lse, ref)


@pytest.mark.parametrize("scale", [0.0, 1.0, 40.0])
def test_scales(ta, scale):
    """Equal weights, and softmaxes that are all but one-hot."""
    c = Cache4([200, 33, 1], 2, 64, 16, seed=5)
    q = torch.randn(3, 6, 64, generator=torch.Generator().manual_seed(2)).to(BF16).cuda()
    for parts in (0, 2):
        check(c, *ta.attn_decode_paged(q, *c.args(), **c.scales(), scale=scale, num_parts=parts), reference(q, c, scale))


def test_bad_lengths_and_pages(ta):
    c = Cache4([40, 20, 16, 50, 64, 33, 7], 2, 128, 16, seed=6)
    q = torch.randn(7, 8, 128, generator=torch.Generator().manual_seed(3)).to(BF16).cuda()
    per = c.table.shape[1]
    c.lens[1], c.lens[2] = -1, per * 16 + 1
    c.table[3, 3], c.table[4, 0] = -7, c.k.shape[0]
    ref = reference(q, c, 0.1)
    assert np.isnan(ref[1][1:5]).all() and np.isfinite(ref[1][[0, 5, 6]]).all()
    for parts in (None, 0, 1, 5, 64):
        check(c, *ta.attn_decode_paged(q, *c.args(), **c.scales(), scale=0.1, num_parts=parts), ref)


@pytest.mark.parametrize("D", [64, 128])
def test_every_group_has_its_own_scale(ta, D):
    """One key at a time (the softmax of one score is 1): O is the value's numbers, for
    scales over the whole range of a bf16 result, groups far apart in one row."""
    g = torch.Generator().manual_seed(D)
    B, P = 64, 16
    codes = torch.randint(0, 256, (2, B, 1, P, D // 2), generator=g, dtype=U8).cuda()
    scales = torch.randint(3, 250, (2, B, 1, P, D // 32), generator=g, dtype=U8)
    scales[0] = 120
    scales = scales.cuda()
    table, lens = torch.arange(B, dtype=torch.int32).view(B, 1).cuda(), torch.ones(B, dtype=torch.int32).cuda()
    q = torch.randn(B, 4, D, generator=g).to(BF16).cuda()
    o, lse = ta.attn_decode_paged(q, codes[0], codes[1], table, lens, k_scale=scales[0], v_scale=scales[1])
    k, v = (ms.mx_values(codes[i].cpu().numpy(), scales[i].cpu().numpy())[:, 0, 0] for i in range(2))
    np.testing.assert_array_equal(f64(o), np.broadcast_to(v[:, None], o.shape))
    want = (f64(q) * k[:, None]).sum(-1) * D ** -0.5
    size = np.abs(f64(q) * k[:, None]).sum(-1) * D ** -0.5
    assert (np.abs(f64(lse) - want) <= (D + 8) * 2.0 ** -24 * size + 2.0 ** -22).all()


@pytest.mark.parametrize("D", [64, 128])
def test_a_nan_scale_within_the_sequence(ta, D):
    """A group whose scale is 255: a key's makes its head NaN, a value's the dims of its
    group; other sequences and heads keep their numbers."""
    c = Cache4([50, 50], 2, D, 16, seed=9)
    q = torch.randn(2, 4, D, generator=torch.Generator().manual_seed(4)).to(BF16).cuda()
    c.scales4[0][c.table[0, 1].long(), 0, 3, 0] = 255
    c.scales4[1][c.table[1, 2].long(), 1, 5, D // 32 - 1] = 255
    for parts in (0, 3):
        o, lse = ta.attn_decode_paged(q, *c.args(), **c.scales(), num_parts=parts)
        bad = torch.zeros(2, 4, D, dtype=torch.bool)
        bad[0, :2] = True
        bad[1, 2:, D - 32:] = True
        assert torch.equal(torch.isnan(o).cpu(), bad)
        assert torch.equal(torch.isnan(lse).cpu(), torch.tensor([[True, True, False, False], [False] * 4]))


def test_pages_past_4_gib(ta):
    """Pages whose byte offset passes 2^32 in the codes of one head."""
    P, D = 1024, 128
    pages = (1 << 32) // (P * D // 2) + 40
    codes = [torch.zeros(pages, 1, P, D // 2, dtype=U8, device="cuda") for _ in range(2)]
    scales = [torch.full((pages, 1, P, D // 32), 255, dtype=U8, device="cuda") for _ in range(2)]
    c = Cache4([2 * P + 100], 1, D, P, seed=8, spare=0, extra=0)
    q = torch.ones(1, 5, D, dtype=BF16, device="cuda")
    ro, rl = ta.attn_decode_paged(q, *c.args(), **c.scales())
    for j, to in enumerate([pages - 1, pages // 2, pages - 30]):
        at = c.table[0, j].long()
        for big, small in zip(codes + scales, c.codes + c.scales4):
            big[to] = small[at]
        c.table[0, j] = to
    o, lse = ta.attn_decode_paged(q, *codes, c.table, c.lens, k_scale=scales[0], v_scale=scales[1])
    assert torch.equal(o, ro) and torch.equal(lse, rl)
