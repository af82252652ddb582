"""GPU parity of qk_norm_rope_append (and of kv_cache_append into 4 bits) against the
float64 oracle.  What the caches take is compared bit for bit: whole caches, so that
anything written beside its place shows.  Queries, and keys in bf16, are within half a
step of bf16 (2^-8) plus 20 roundings of fp32 (2^-24 each) of the two products that
make them: the mean of squares (8 a lane, then 3 or 4 levels of the tree, halved by the
root), the root, quotient and two products of the norm, two products and their sum."""
import numpy as np
import pytest

from oracle import more_serving as ms
from oracle import serving

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, F32, E4M3, U8, I32 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.uint8, torch.int32


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
    return t.contiguous().view(U8 if t.element_size() == 1 else torch.int16).cpu().numpy()


def bf16_bits(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(BF16).view(torch.int16).numpy()


class Pool:
    """A paged cache of one type, full of a pattern, with its scales and its table."""

    def __init__(self, B, per, Hkv, D, P, kind, seed=0):
        g = torch.Generator().manual_seed(seed)
        pages = B * per + 3
        self.table = torch.randperm(pages, generator=g)[:B * per].to(I32).view(B, per).cuda()
        shape = (pages, Hkv, P, D)
        self.kind, self.ks, self.vs = kind, None, None
        if kind == "mxfp4":
            rand = lambda *s: torch.randint(0, 255, s, generator=g, dtype=U8).cuda()   # noqa: E731
            self.k, self.v = rand(*shape[:3], D // 2), rand(*shape[:3], D // 2)
            self.ks, self.vs = rand(*shape[:3], D // 32), rand(*shape[:3], D // 32)
        else:
            self.k, self.v = (torch.randn(shape, generator=g).to(BF16).cuda() for _ in range(2))
            if kind == "e4m3":
                self.k, self.v = self.k.to(E4M3), self.v.to(E4M3)
                self.ks, self.vs = (s.contiguous().cuda() for s in ((torch.rand(2, Hkv, generator=g) + 0.5) / 60).unbind(0))

    def tensors(self):
        return (self.k, self.v) + ((self.ks, self.vs) if self.kind == "mxfp4" else ())

    def want(self, new, scale, which, pos, seq, held):
        """The arrays after the append of float64 rows `new` [T, Hkv, D] where `held`."""
        cache = bits((self.k, self.v)[which])
        out = [cache.copy()] + ([bits((self.ks, self.vs)[which]).copy()] if self.kind == "mxfp4" else [])
        table, (pages, _, P) = self.table.cpu().numpy(), cache.shape[:3]
        for t in range(len(new)):
            at = serving.place(table, pages, P, t if seq is None else int(seq[t]), int(pos[t])) if held[t] else None
            if at is None:
                continue
            if self.kind == "mxfp4":
                out[0][at[0], :, at[1]], out[1][at[0], :, at[1]] = ms.mx_pack(new[t].astype(np.float32))
            elif self.kind == "e4m3":
                s = scale.cpu().numpy().astype(np.float64)
                out[0][at[0], :, at[1]] = serving.e4m3_codes((new[t] / s[:, None]).astype(np.float32))
            else:
                out[0][at[0], :, at[1]] = bf16_bits(new[t])
        return out


def angles(rows, rot):
    a = np.arange(rows)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / rot)
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)).cuda()


CASES = [
    # (T, B, Hq, Hkv, D, page, norms, rot, interleaved, seq given)
    (1, 1, 1, 1, 64, 16, "", 64, False, False),
    (1, 3, 8, 2, 128, 16, "qk", 128, False, True),
    (5, 7, 3, 1, 64, 32, "q", 32, True, False),
    (33, 3, 5, 5, 128, 64, "k", 48, False, True),
    (33, 3, 5, 5, 128, 64, "", 16, True, True),
    (70, 2, 16, 4, 64, 16, "qk", 48, False, True),
    (64, 64, 32, 8, 128, 256, "qk", 0, False, False),
    (1100, 5, 7, 3, 64, 64, "qk", 64, True, True),
    (1500, 4, 32, 8, 128, 64, "qk", 112, False, True),
]


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "mxfp4"])
def test_against_oracle(ta, case, kind):
    T, B, Hq, Hkv, D, P, norms, rot, inter, given = case
    g = torch.Generator().manual_seed(T + D)
    top = -(-T // B) + 40
    pool = Pool(B, -(-top // P) + 1, Hkv, D, P, kind, seed=T)
    qkv = torch.randn(T, Hq + 2 * Hkv + 1, D, generator=g).to(BF16).cuda()
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:Hq + 2 * Hkv]
    seq = torch.arange(T, dtype=I32) % B
    pos = (torch.arange(T, dtype=I32) // B) + torch.randint(0, 40, (B,), generator=g)[seq.long()].to(I32)
    rows = int(pos.max()) + 1
    if T > 5:   # padding; past the table; past the angles; a page, a sequence that is not there
        pos[1], pos[2], pos[3] = -1, pool.table.shape[1] * P, 2 ** 31 - 1
        rows = pool.table.shape[1] * P + 1
        pool.table[B - 1, 0] = pool.k.shape[0]
        if given:
            seq[0], seq[4] = -1, B
    cos_sin = angles(rows, rot) if rot else None
    w = [(torch.randn(D, generator=g) * 0.2 + 1).to(BF16).cuda() if n in norms else None for n in "qk"]
    pn, sn = pos.numpy(), seq.numpy() if given else None
    turned = (pn >= 0) & (pn < rows) if rot else pn >= 0
    at = np.where(turned, pn, 0)
    cs = cos_sin.cpu().numpy() if rot else None
    y = [ms.norm_rope(f64(x), at, None if n is None else f64(n), 1e-5, cs, inter) for x, n in ((q, w[0]), (k, w[1]))]
    tol = [20 * 2.0 ** -24 * size + 2.0 ** -8 * np.abs(x) for x, size in y]
    want_k, want_v = (pool.want(x, s, i, pn, sn, turned) for i, (x, s) in enumerate(((y[1][0], pool.ks), (f64(v), pool.vs))))

    out = torch.full((T, Hq, D), 7.0, dtype=BF16, device="cuda")
    r = ta.qk_norm_rope_append(q, k, v, pool.k, pool.v, pool.table, pos.cuda(), cos_sin=cos_sin, q_weight=w[0],
                               k_weight=w[1], eps=1e-5, interleaved=inter, seq=seq.cuda() if given else None,
                               k_scale=pool.ks, v_scale=pool.vs, out=out)
    assert r[0] is out and r[1] is pool.k and r[2] is pool.v
    got = f64(out)
    assert (got[pn < 0] == 0).all()
    if rot:
        assert np.isnan(got[pn >= rows]).all()
    err = np.abs(got[turned] - y[0][0][turned])
    print(f"  queries: {(err / tol[0][turned]).max():.2f} of bound", flush=True)
    assert (err <= tol[0][turned]).all()
    if kind == "bf16":
        new, old = torch.from_numpy(want_k[0]).view(BF16).double().numpy(), f64(pool.k)
        lim = np.zeros_like(new)            # where the append went, the key's bound; elsewhere none
        for t in range(T):
            to = serving.place(pool.table.cpu().numpy(), len(new), P, t if sn is None else int(sn[t]), int(pn[t])) if turned[t] else None
            if to is not None:
                lim[to[0], :, to[1]] = tol[1][t] + 2.0 ** -8 * np.abs(y[1][0][t])   # (new is itself rounded)
        assert (np.abs(new - old) <= lim).all()
    else:
        for a, b in zip(want_k, (pool.k, pool.ks)):
            np.testing.assert_array_equal(bits(b), a)
    for a, b in zip(want_v, (pool.v, pool.vs)):
        np.testing.assert_array_equal(bits(b), a)


@pytest.mark.parametrize("rope", [False, True], ids=["append", "rope"])
def test_every_bf16_number_into_4_bits(ta, rope):
    """Ties, the scales' steps, denormals, zeros of both signs, infinities, NaN; in the
    order of the numbers, shuffled, and a group at a time."""
    x = torch.arange(1 << 16, dtype=I32).to(torch.int16)
    x = torch.cat([x, x[torch.randperm(1 << 16, generator=torch.Generator().manual_seed(1))]])
    finite = x[:1 << 16][(x[:1 << 16] & 0x7F80) != 0x7F80]
    order = finite[torch.randperm(len(finite), generator=torch.Generator().manual_seed(2))][:60 * 1024]
    x = torch.cat([x, order]).view(BF16)
    T = len(x) // 128
    x = x.view(T, 1, 128).cuda()
    P = 16
    pool = Pool(1, -(-T // P), 1, 128, P, "mxfp4", seed=3)
    pos, seq = torch.arange(T, dtype=I32, device="cuda"), torch.zeros(T, dtype=I32, device="cuda")
    wk, wv = (pool.want(f64(x).astype(np.float32), None, i, pos.cpu().numpy(), seq.cpu().numpy(), [True] * T) for i in range(2))
    if rope:    # without weights and angles: the numbers as they are
        out, _, _ = ta.qk_norm_rope_append(x, x, x, pool.k, pool.v, pool.table, pos, seq=seq, k_scale=pool.ks, v_scale=pool.vs)
        fin = ~torch.isnan(x)
        assert torch.equal(out.view(torch.int16)[fin], x.view(torch.int16)[fin]) and torch.isnan(out[~fin]).all()
    else:
        ta.kv_cache_append(x, x, pool.k, pool.v, pool.table, pos, seq=seq, k_scale=pool.ks, v_scale=pool.vs)
    for a, b in zip(wk + wv, (pool.k, pool.ks, pool.v, pool.vs)):
        np.testing.assert_array_equal(bits(b), a)


@pytest.mark.parametrize("kind", ["bf16", "mxfp4"])
def test_norm_of_zeros_infinities_and_nan(ta, kind):
    """A head of zeros stays zeros; an infinity in a head makes the others of it 0 and
    itself NaN (inf / inf), and by the rotation its partner too (NaN times a sine of 0); a
    NaN makes the head NaN; other heads keep their numbers, large ones are normed."""
    T, D = 6, 64
    x = torch.ones(T, 2, D, dtype=BF16)
    x[0], x[1, 0, 3], x[2, 1, 5], x[3], x[4] = 0, float("inf"), float("nan"), 1e15, 1e-30
    x = x.cuda()
    w = torch.ones(D, dtype=BF16, device="cuda")
    pool = Pool(T, 1, 2, D, 16, kind, seed=4)
    pos = torch.zeros(T, dtype=I32, device="cuda")
    out, kc, _ = ta.qk_norm_rope_append(x, x, x, pool.k, pool.v, pool.table, pos, q_weight=w, k_weight=w, eps=0.0 if kind == "bf16" else 1e-6,
                                        cos_sin=angles(1, 64), k_scale=pool.ks, v_scale=pool.vs)
    o = f64(out)
    assert (o[0] == 0).all() if kind == "mxfp4" else np.isnan(o[0]).all()      # (0 / 0 without eps)
    assert np.isnan(o[1, 0, [3, 35]]).all() and (np.delete(o[1, 0], [3, 35]) == 0).all() and (o[1, 1] == 1).all()
    assert np.isnan(o[2, 1]).all() and (o[2, 0] == 1).all() and (o[3] == 1).all() and (o[5] == 1).all()
    if kind == "mxfp4":
        page = pool.table[:, 0].long()
        held = ms.mx_values(bits(kc[page, :, 0]), bits(pool.ks[page, :, 0]))
        assert (held[0] == 0).all() and np.isnan(held[1, 0]).all() and np.isnan(held[2, 1]).all()
        assert (held[1, 1] == 1).all() and (held[3] == 1).all() and (held[5] == 1).all()


def test_far_positions_and_pages_past_4_gib(ta):
    """Rows of the caches whose byte offset passes 2^32, and of cos_sin past 2^31."""
    P, D = 1024, 128
    pages = (1 << 32) // (P * D * 2) + 3
    k, v = (torch.zeros(pages, 1, P, D, dtype=BF16, device="cuda") for _ in range(2))
    rows = (1 << 31) // (128 * 4) + 5000
    cs = torch.zeros(rows, 128, device="cuda")
    cs[rows - 1, :64], cs[rows - 1, 64:] = 0.5, 2.0
    table = torch.full((1, -(-rows // P)), -1, dtype=I32, device="cuda")
    table[0, (rows - 1) // P] = pages - 1
    x = torch.ones(1, 1, D, dtype=BF16, device="cuda")
    out, _, _ = ta.qk_norm_rope_append(x, x, x, k, v, table, torch.tensor([rows - 1], dtype=I32, device="cuda"), cos_sin=cs)
    want = torch.cat([torch.full((64,), -1.5), torch.full((64,), 2.5)])
    assert torch.equal(out[0, 0].float().cpu(), want)
    at = (pages - 1, 0, (rows - 1) % P)
    assert torch.equal(k[at].float().cpu(), want) and (v[at] == 1).all()
    assert int((k != 0).sum()) == D and int((v != 0).sum()) == D
