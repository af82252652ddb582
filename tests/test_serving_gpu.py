"""GPU parity of the serving step's calls (kv_cache_append, attn_decode_paged,
gemm_bf16_epilogue) against the float64 oracle, through the binding.  Tolerances
are the oracle's bounds for fp32 arithmetic on exact bf16 products, plus half a
step (2^-8 of the value) for a bf16 result and 2^-15 of the largest |V| for the
16-bit softmax weights behind a bf16 O.  The caches' unused rows and pages hold
NaN and the table's unused entries point outside, so that anything read past a
sequence's end shows."""
import numpy as np
import pytest

from oracle import serving
from paper_2504_17577_amd import gen

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def ta():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2504_17577_amd import tileattn
    tileattn.lib()
    return tileattn


def f64(t):
    return t.double().cpu().numpy()


def bits(t):
    return t.contiguous().view(torch.uint8 if t.dtype == E4M3 else torch.int16).cpu().numpy()


class Cache:
    """A pool with every sequence's pages in random order and NaN everywhere no
    sequence has a position; table entries past a sequence's last page are bad."""

    def __init__(self, lens, Hkv, D, P, e4m3=False, seed=0, spare=3, extra=2):
        g = torch.Generator().manual_seed(seed)
        B = len(lens)
        need = [-(-n // P) for n in lens]
        per = max(1, max(need)) + extra
        pages = sum(need) + spare
        order = torch.randperm(pages, generator=g).tolist()
        table = torch.tensor([-1, 2 ** 31 - 1, pages, -2 ** 31], dtype=torch.int32).repeat(B * per)[:B * per].view(B, per)
        held = torch.zeros(pages, P, dtype=torch.bool)
        for b in range(B):
            for j in range(need[b]):
                table[b, j] = order.pop()
                held[table[b, j], :max(0, min(P, lens[b] - j * P))] = True
        shape = (pages, Hkv, P, D)
        self.k_scale = self.v_scale = None
        out = []
        for _ in range(2):
            x = torch.randn(shape, generator=g)
            x = (x * 100).clamp(-448, 448).to(E4M3) if e4m3 else x.to(BF16)
            nan = torch.tensor(float("nan")).to(x.dtype)
            if e4m3:
                x = torch.where(held[:, None, :, None], x.view(torch.uint8), nan.view(torch.uint8)).view(E4M3)
            else:
                x = torch.where(held[:, None, :, None], x, nan)
            out.append(x.cuda())
        self.k, self.v = out
        if e4m3:
            self.k_scale, self.v_scale = ((torch.rand(2, Hkv, generator=g) + 0.5) / 100).cuda().unbind(0)
            self.k_scale, self.v_scale = self.k_scale.contiguous(), self.v_scale.contiguous()
        self.table, self.lens = table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()

    def args(self):
        return self.k, self.v, self.table, self.lens

    def scales(self):
        return dict(k_scale=self.k_scale, v_scale=self.v_scale)


def reference(q, c, scale):
    sc = [None if s is None else f64(s) for s in (c.k_scale, c.v_scale)]
    return serving.attn_paged(f64(q), f64(c.k), f64(c.v), c.table.cpu().numpy(), c.lens.tolist(), scale, *sc)


def check(c, o, lse, ref):
    ro, rl, tol, tol_lse = ref
    o16 = o.dtype == BF16
    got, gl = f64(o), f64(lse)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(ro))
    np.testing.assert_array_equal(np.isfinite(gl), np.isfinite(rl))
    fin = np.isfinite(rl)
    top = np.abs(np.nan_to_num(f64(c.v))).max() * (1 if c.v_scale is None else float(c.v_scale.max()))
    tol = tol[:, :, None] + (2.0 ** -8 * np.abs(ro) + 2.0 ** -15 * top if o16 else 0)
    eo, el = np.abs(got[fin] - ro[fin]), np.abs(gl[fin] - rl[fin])
    assert (got[rl == -np.inf] == 0).all()
    if fin.any():
        print(f"  max|dO| {eo.max():.2e} (of bound {(eo / tol[fin]).max():.2f}) max|dLSE| {el.max():.2e}", flush=True)
        assert (eo <= tol[fin]).all() and (el <= tol_lse[fin]).all()


ATTN = [
    # (lens, Hq, Hkv, D, page, e4m3)
    ([1], 1, 1, 64, 16, False),
    ([0], 4, 2, 128, 16, False),
    ([37], 8, 2, 64, 16, False),
    ([16, 17, 31, 32, 33, 15, 0, 1], 4, 4, 128, 16, False),
    ([63, 64, 65, 127, 128, 129, 500, 2], 8, 2, 128, 64, False),
    ([300, 5], 3, 1, 64, 32, False),
    ([1000, 0, 0, 999, 17], 32, 8, 128, 256, False),
    ([130, 77], 16, 1, 128, 16, False),      # a full tile of rows
    ([130, 77], 17, 1, 64, 16, False),       # one more
    ([257, 31], 48, 1, 128, 32, False),
    ([100, 700], 64, 2, 64, 1024, False),
    ([4099, 1, 2500], 8, 8, 64, 64, False),
    ([40], 128, 1, 128, 16, False),
    ([1, 0, 37], 4, 2, 64, 16, True),
    ([16, 17, 33, 129], 8, 2, 128, 16, True),
    ([1500, 64, 63], 16, 1, 128, 64, True),
    ([513, 2], 40, 2, 64, 128, True),
    ([9001], 8, 2, 128, 64, True),
    (list(range(70)), 2, 2, 64, 16, False),  # more sequences than lanes, most of them short
    ([7 * i % 90 for i in range(300)], 4, 2, 64, 16, False),
]


@pytest.mark.parametrize("case", ATTN, ids=[f"{len(c[0])}x{max(c[0])}-h{c[1]}.{c[2]}-d{c[3]}-p{c[4]}{'-e4m3' * c[5]}" for c in ATTN])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
def test_attention_against_oracle(ta, case, dtype):
    lens, Hq, Hkv, D, P, e4m3 = case
    c = Cache(lens, Hkv, D, P, e4m3, seed=len(lens))
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
def test_attention_scales(ta, scale):
    """Equal weights, and softmaxes that are all but one-hot."""
    c = Cache([200, 33, 1], 2, 64, 16, seed=5)
    q = torch.randn(3, 6, 64, generator=torch.Generator().manual_seed(2)).to(BF16).cuda()
    for parts in (0, 2):
        check(c, *ta.attn_decode_paged(q, *c.args(), scale=scale, num_parts=parts), reference(q, c, scale))


def test_attention_of_bad_lengths_and_pages(ta):
    """A length outside the table and a page outside the pool give NaN in their
    sequence alone; nothing outside is read (the kernel's own checks)."""
    c = Cache([40, 20, 16, 50, 64, 33, 7], 2, 128, 16, seed=6)
    q = torch.randn(7, 8, 128, generator=torch.Generator().manual_seed(3)).to(BF16).cuda()
    per = c.table.shape[1]
    c.lens[1], c.lens[2] = -1, per * 16 + 1
    c.table[3, 3], c.table[4, 0] = -7, c.k.shape[0]
    ref = reference(q, c, 0.1)
    assert np.isnan(ref[1][1:5]).all() and np.isfinite(ref[1][[0, 5, 6]]).all()
    for parts in (None, 0, 1, 5, 64):
        check(c, *ta.attn_decode_paged(q, *c.args(), scale=0.1, num_parts=parts), ref)


def test_sequences_that_share_pages(ta):
    c = Cache([64, 48, 33], 2, 64, 16, seed=7)
    c.table[1, :2], c.table[2, :2] = c.table[0, :2], c.table[0, :2]
    q = torch.randn(3, 4, 64, generator=torch.Generator().manual_seed(4)).to(BF16).cuda()
    check(c, *ta.attn_decode_paged(q, *c.args()), reference(q, c, 0.125))


def test_attention_past_4_gib(ta):
    """Pages whose byte offset passes 2^32 in a cache of one head."""
    P, D = 1024, 128
    pages = (1 << 32) // (P * D * 2) + 40
    kc, vc = (torch.zeros(pages, 1, P, D, dtype=BF16, device="cuda") for _ in range(2))
    c = Cache([2 * P + 100], 1, D, P, seed=8, spare=0, extra=0)
    for j, to in enumerate([pages - 1, pages // 2, pages - 30]):
        kc[to], vc[to] = c.k[c.table[0, j].long()], c.v[c.table[0, j].long()]
        c.table[0, j] = to
    o, lse = ta.attn_decode_paged(torch.ones(1, 5, D, dtype=BF16, device="cuda"), kc, vc, c.table, c.lens)
    small = Cache([2 * P + 100], 1, D, P, seed=8, spare=0, extra=0)
    ro, rl = ta.attn_decode_paged(torch.ones(1, 5, D, dtype=BF16, device="cuda"), *small.args())
    assert torch.equal(o, ro) and torch.equal(lse, rl)


APPEND = [
    # (T, B, Hkv, D, page, e4m3, seq given)
    (1, 1, 1, 64, 16, False, False),
    (5, 7, 2, 128, 16, False, False),
    (33, 3, 3, 64, 32, False, True),
    (700, 5, 8, 128, 64, False, True),
    (1, 1, 1, 64, 16, True, True),
    (6, 6, 4, 128, 16, True, False),
    (257, 4, 5, 64, 256, True, True),
]


def tokens(T, Hkv, D, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(T, 3 * Hkv + 1, D, generator=g).to(BF16).cuda()


@pytest.mark.parametrize("case", APPEND, ids=[str(c) for c in APPEND])
def test_append_against_oracle(ta, case):
    T, B, Hkv, D, P, e4m3, given = case
    g = torch.Generator().manual_seed(T)
    top = -(-T // B) + 40
    c = Cache([top] * B, Hkv, D, P, e4m3, seed=T)
    qkv = tokens(T, Hkv, D, T)
    k, v = qkv[:, Hkv:2 * Hkv], qkv[:, 2 * Hkv:3 * Hkv]
    seq = torch.arange(T, dtype=torch.int32) % B
    pos = (torch.arange(T, dtype=torch.int32) // B) + torch.randint(0, 40, (B,), generator=g)[seq.long()].to(torch.int32)
    if T > 4:   # padding, past the table, a page that is not there, a sequence that is not
        pos[1], pos[2] = -1, c.table.shape[1] * P
        c.table[B - 1, 0] = c.k.shape[0]
        if given:
            seq[0], seq[4] = -1, B
    table, kind = c.table.cpu().numpy(), np.uint8 if e4m3 else np.uint16
    want = [serving.append(bits(n).view(np.uint16), bits(x).view(kind), table, pos.numpy(), seq.numpy() if given else None,
                           None if s is None else s.cpu().numpy())
            for n, x, s in ((k, c.k, c.k_scale), (v, c.v, c.v_scale))]
    r = ta.kv_cache_append(k, v, c.k, c.v, c.table, pos.cuda(), seq=seq.cuda() if given else None, **c.scales())
    assert r[0] is c.k and r[1] is c.v
    for got, w in zip((c.k, c.v), want):
        np.testing.assert_array_equal(bits(got).view(kind), w)


@pytest.mark.parametrize("scale", [None, 1.0, 0.37, 2.0 ** -7, 3e-39, 0.0])
def test_append_of_every_bf16_number_to_e4m3(ta, scale):
    """Ties, the ends of the range, denormal quotients, infinities; NaN stays NaN."""
    x = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(BF16).view(1 << 9, 1, 128).cuda()
    kc, vc = (torch.zeros(32, 1, 16, 128, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
    table = torch.arange(32, dtype=torch.int32, device="cuda").view(1, 32)
    pos = torch.arange(512, dtype=torch.int32, device="cuda")
    s = None if scale is None else torch.tensor([scale], device="cuda")
    ta.kv_cache_append(x, x, kc, vc, table, pos, seq=torch.zeros_like(pos), k_scale=s, v_scale=s)
    with np.errstate(all="ignore"):
        q = (bits(x).view(np.uint16).astype(np.uint32) << 16).view(np.float32) / np.float32(1 if scale is None else scale)
    want = serving.e4m3_codes(q).reshape(-1)
    for c in (kc, vc):
        got, nan = bits(c).reshape(-1), np.isnan(q).reshape(-1)
        np.testing.assert_array_equal(got[~nan], want[~nan])
        assert (got[nan] & 0x7F == 0x7F).all()


GEMM = [
    # (M, N, K)
    (1, 8, 8), (1, 4096, 4096), (1, 72, 1000), (2, 64, 64), (5, 136, 264), (16, 128, 512), (17, 1000, 1032),
    (24, 2048, 1024), (32, 256, 4096), (33, 520, 72), (48, 4096, 256), (64, 136, 2056), (65, 200, 520),
    (96, 1024, 1024), (127, 136, 128), (128, 128, 64), (129, 264, 328), (200, 1000, 1000), (256, 256, 256),
    (300, 8, 40), (389, 520, 1032), (513, 1032, 200),
]
EPILOGUE = [("none", 0, 0), ("relu", 1, 0), ("gelu", 1, 1), ("gelu_tanh", 0, 1), ("silu", 1, 1), ("none", 1, 1)]


@pytest.mark.parametrize("M,N,K", GEMM)
def test_gemm_against_oracle(ta, M, N, K):
    g = torch.Generator().manual_seed(M + N + K)
    a = torch.randn(M, K, generator=g).to(BF16).cuda()
    b = (torch.randn(K, N, generator=g) * K ** -0.5).to(BF16).cuda()
    bias, res = torch.randn(N, generator=g).to(BF16).cuda(), torch.randn(M, N, generator=g).cuda()
    for i, (act, has_bias, has_res) in enumerate(EPILOGUE):
        dt = F32 if i % 2 == (M % 2) else BF16
        r = res.to(dt) if has_res else None
        c, tol = serving.gemm_epilogue(f64(a), f64(b), f64(bias) if has_bias else None, act, f64(r) if has_res else None)
        if dt == BF16:
            tol = tol + 2.0 ** -8 * np.abs(c)
        for splits in (None, 1, 2, 7):
            got = ta.gemm_bf16_epilogue(a, b, bias=bias if has_bias else None, activation=act, residual=r, out_dtype=dt,
                                        num_splits=splits)
            assert got.dtype == dt and got.shape == (M, N)
            err = np.abs(f64(got) - c)
            print(f"  {act} {has_bias} {has_res} {dt} splits {splits}: max error {err.max():.2e}, of bound "
                  f"{(err / tol).max():.2f}", flush=True)
            assert (err <= tol).all()


@pytest.mark.parametrize("M,N,K", [(4096, 4096, 64), (4100, 4104, 72), (4096, 4360, 136), (2000, 16392, 200), (8200, 2050 * 4, 64)])
def test_gemm_in_large_tiles(ta, M, N, K):
    """Products with whole rounds of 256 x 256 tiles and other columns after them, the
    oracle's arithmetic on the GPU (float64)."""
    g = torch.Generator(device="cuda").manual_seed(N)
    a, b = torch.randn(M, K, generator=g, device="cuda").to(BF16), torch.randn(K, N, generator=g, device="cuda").to(BF16)
    bias, r = torch.randn(N, generator=g, device="cuda").to(BF16), torch.randn(M, N, generator=g, device="cuda").to(BF16)
    x = a.double() @ b.double() + bias.double()
    size = a.double().abs() @ b.double().abs() + bias.double().abs()
    y = x * torch.sigmoid(x)
    # as oracle.serving.gemm_epilogue's, and half a step of bf16
    tol = 1.13 * (K + 2) * 2.0 ** -24 * size + 2.0 ** -20 * y.abs() + (2.0 ** -24 + 2.0 ** -8) * (y + r.double()).abs() + 1e-30
    for splits in (None, 1, 3):
        got = ta.gemm_bf16_epilogue(a, b, bias=bias, activation="silu", residual=r, out_dtype=BF16, num_splits=splits)
        err = (got.double() - y - r.double()).abs()
        print(f"  splits {splits}: of bound {float((err / tol).max()):.2f}", flush=True)
        assert (err <= tol).all()


@pytest.mark.parametrize("M", [1, 40, 300])
@pytest.mark.parametrize("dt", [F32, BF16], ids=["fp32", "bf16"])
def test_gemm_onto_the_residual_in_place(ta, M, dt):
    g = torch.Generator().manual_seed(M)
    a, b = torch.randn(M, 520, generator=g).to(BF16).cuda(), (torch.randn(520, 264, generator=g) / 20).to(BF16).cuda()
    x = torch.randn(M, 264, generator=g).to(dt).cuda()
    for splits in (1, 3):
        y = x.clone()
        want = ta.gemm_bf16_epilogue(a, b, residual=x, out_dtype=dt, num_splits=splits)
        assert ta.gemm_bf16_epilogue(a, b, residual=y, out=y, out_dtype=dt, num_splits=splits) is y
        assert torch.equal(y, want)


@pytest.mark.parametrize("M", [1, 20, 100, 300])
def test_gemm_of_infinities_and_nan(ta, M):
    """What a row or column of A or B holds stays in that row or column of C."""
    a = torch.ones(M, 136, dtype=BF16, device="cuda")
    b = torch.ones(136, 200, dtype=BF16, device="cuda")
    a[M - 1, 135], b[135, 199], b[0, 7] = float("inf"), float("nan"), float("-inf")
    c = ta.gemm_bf16_epilogue(a, b)
    want = torch.full((M, 200), 136.0)
    want[:, 7] = float("-inf")
    want[M - 1] = float("inf")
    want[M - 1, 7] = float("nan")
    want[:, 199] = float("nan")
    np.testing.assert_array_equal(c.cpu().numpy(), want.numpy())


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_activations_over_their_range(ta, act):
    """Every bf16 number from 2^-20 to 2^7 and its negative, by a product with one:
    relative to the value, where 1 + tanh and 1 + erf cancel too."""
    x = torch.arange(0x3580, 0x4300, dtype=torch.int32).to(torch.int16).view(BF16)
    x = torch.cat([x, -x]).view(-1, 1)
    a = torch.zeros(x.shape[0], 8, dtype=BF16)
    a[:, :1] = x
    b = torch.zeros(8, 8, dtype=BF16)
    b[0] = 1
    got = ta.gemm_bf16_epilogue(a.cuda(), b.cuda(), activation=act)[:, 0].double().cpu()
    y = x[:, 0].double()
    want = {"relu": y.clamp(min=0), "gelu": 0.5 * y * torch.erfc(-y / 2 ** 0.5), "silu": y * torch.sigmoid(y),
            "gelu_tanh": y * torch.sigmoid(2 * (2 / np.pi) ** 0.5 * (y + 0.044715 * y ** 3))}[act]
    # 2^-20 of the value, and the argument's own rounding (2^-23 of |x^3| or x^2 at most) in the exponent;
    # where 1 + exp(-u) passes 2^126 its reciprocal is below fp32's smallest normal number, and the
    # result 0 where it is x exp(u) < 2^7 2^-126
    tol = want.abs() * (2.0 ** -20 + 2.0 ** -22 * (1 + y.abs() ** 3).clamp(max=100)) + 2.0 ** -119
    assert ((got - want).abs() <= tol).all()
