"""The serving step on 4-bit numbers, its calls together: a decoder whose weights and
caches are MXFP4, from the projection over norm, rotation and append, attention, output
projection and MLP to the logits and the next token, which the next step's input is
made of.  Each call is held to the oracle on the inputs that it got; a captured step,
replayed with other tokens, positions and wishes, to the same step run eagerly, bit for
bit; and the step on two streams at once, and with workspaces of its own, to itself."""
import numpy as np
import pytest

from oracle import more_serving as ms
from oracle import serving

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, F32, U8, I32 = torch.bfloat16, torch.float32, torch.uint8, torch.int32


@pytest.fixture(scope="module")
def ta():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2504_17577_amd import tileattn
    tileattn.lib()
    return tileattn


def f64(t):
    return t.double().cpu().numpy()


class Decoder:
    """Two layers and a head for a batch of five slots."""
    HID, HQ, HKV, D, FF, V, B, P, PER = 256, 6, 2, 64, 512, 1000, 5, 16, 6

    def __init__(self, ta, seed=0):
        self.ta, g = ta, torch.Generator().manual_seed(seed)

        def weight(n, k, std):
            c, s = ms.mx_pack((torch.randn(n, k, generator=g) * std).numpy())
            return torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()

        n = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(BF16).cuda()   # noqa: E731
        heads = self.HQ + 2 * self.HKV
        self.embed = n(self.V, self.HID)
        self.head = weight(self.V, self.HID, 0.15)
        pages = self.B * self.PER + 3
        self.table = torch.randperm(pages, generator=g)[:self.B * self.PER].to(I32).view(self.B, self.PER).cuda()
        cache = lambda d: torch.full((pages, self.HKV, self.P, d), 255, dtype=U8, device="cuda")   # noqa: E731  (NaN)
        self.layers = [dict(wqkv=weight(heads * self.D, self.HID, self.HID ** -0.5), bqkv=n(heads * self.D, std=0.3),
                            qw=n(self.D, std=0.2) + 1, kw=n(self.D, std=0.2) + 1, wo=weight(self.HID, self.HQ * self.D, 0.05),
                            w1=weight(self.FF, self.HID, 0.06), b1=n(self.FF, std=0.3), w2=weight(self.HID, self.FF, 0.04),
                            kc=cache(self.D // 2), vc=cache(self.D // 2), ks=cache(self.D // 32), vs=cache(self.D // 32))
                       for _ in range(2)]
        a = np.arange(self.P * self.PER)[:, None] * 10000.0 ** (-np.arange(0, self.D, 2) / self.D)
        self.cos_sin = torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)).cuda()

    def clone(self):
        other = object.__new__(Decoder)
        other.__dict__.update(self.__dict__)
        other.layers = [dict(lay, **{n: lay[n].clone() for n in ("kc", "vc", "ks", "vs")}) for lay in self.layers]
        return other

    def step(self, tokens, seq, pos, lens, wish, seen=None, stream=None):
        """One pass over tokens [T] at positions pos of sequences seq (None: one a slot)."""
        ta, T, s = self.ta, tokens.shape[0], dict(stream=stream)
        x = self.embed[tokens.clamp(min=0).long()]
        for lay in self.layers:
            qkv = ta.gemm_mxfp4_epilogue(x, *lay["wqkv"], bias=lay["bqkv"], out_dtype=BF16, **s).view(T, -1, self.D)
            q, k, v = qkv[:, :self.HQ], qkv[:, self.HQ:self.HQ + self.HKV], qkv[:, self.HQ + self.HKV:]
            sc = dict(k_scale=lay["ks"], v_scale=lay["vs"])
            qr, _, _ = ta.qk_norm_rope_append(q, k, v, lay["kc"], lay["vc"], self.table, pos, cos_sin=self.cos_sin,
                                              q_weight=lay["qw"], k_weight=lay["kw"], seq=seq, **sc, **s)
            if seq is not None:
                continue   # a prefill's attention is not what is looked at here
            o, lse = ta.attn_decode_paged(qr, lay["kc"], lay["vc"], self.table, lens, out_dtype=BF16, **sc, **s)
            mid = ta.gemm_mxfp4_epilogue(o.view(T, -1), *lay["wo"], residual=x, out_dtype=BF16, **s)
            h = ta.gemm_mxfp4_epilogue(mid, *lay["w1"], bias=lay["b1"], activation="silu", out_dtype=BF16, **s)
            out = ta.gemm_mxfp4_epilogue(h, *lay["w2"], residual=mid, out_dtype=BF16, **s)
            if seen is not None:
                seen.append(dict(lay=lay, x=x, qkv=qkv, q=q, k=k, v=v, qr=qr, o=o, lse=lse, mid=mid, h=h, out=out,
                                 **{n: lay[n].clone() for n in ("kc", "vc", "ks", "vs")}))
            x = out
        if seq is not None:
            return None
        logits = ta.gemm_mxfp4_epilogue(x, *self.head, out_dtype=BF16, **s)
        token, logp = ta.sample_logits(logits, **wish, **s)
        return logits, token, logp

    def prefill(self, lens, seed=1):
        g = torch.Generator().manual_seed(seed)
        seq = torch.tensor([b for b, n in enumerate(lens) for _ in range(n)] + [0, 3], dtype=I32, device="cuda")
        pos = torch.tensor([t for n in lens for t in range(n)] + [-1, -1], dtype=I32, device="cuda")
        self.step(torch.randint(0, self.V, (len(seq),), generator=g).cuda(), seq, pos, None, None)

    def wish(self, seed):
        g = torch.Generator().manual_seed(seed)
        return dict(u=torch.rand(self.B, generator=g).cuda(), temperature=torch.tensor([0.7, 0.0, 1.0, 1.3, 0.9]).cuda(),
                    top_k=torch.tensor([40, 0, 5, 0, 600], dtype=I32).cuda(), top_p=torch.tensor([0.9, 0.5, 1.0, 0.95, 0.8]).cuda(),
                    min_p=torch.tensor([0.0, 0.1, 0.0, 0.01, 0.05]).cuda())


def close(got, want, tol):
    err = np.abs(f64(got).reshape(want.shape) - want)
    assert (err <= tol + 2.0 ** -8 * np.abs(want)).all(), float((err / (tol + 2.0 ** -8 * np.abs(want))).max())


def product(x, w, *args, **kw):
    return serving.gemm_epilogue(x, ms.mx_values(w[0].cpu().numpy(), w[1].cpu().numpy()).T, *args, **kw)


def test_step_against_oracle(ta):
    d = Decoder(ta)
    held = [0, 15, 16, 0, 77]                       # slot 3 stays idle
    d.prefill(held)
    tokens = torch.tensor([3, 1, 4, 0, 9], device="cuda")
    live = [0, 1, 2, 4]
    for step in range(3):
        pos = torch.tensor([n + step if b != 3 else -1 for b, n in enumerate(held)], dtype=I32, device="cuda")
        before = d.clone().layers
        seen, wish = [], d.wish(step)
        logits, token, logp = d.step(tokens, None, pos, pos + 1, wish, seen)
        pn, table = pos.cpu().numpy(), d.table.cpu().numpy()
        for s, old in zip(seen, before):
            lay = s["lay"]
            close(s["qkv"].reshape(5, -1), *product(f64(s["x"]), lay["wqkv"], f64(lay["bqkv"])))
            at = np.maximum(pn, 0)
            y = [ms.norm_rope(f64(s[n]), at, f64(lay[w]), 1e-6, d.cos_sin.cpu().numpy()) for n, w in (("q", "qw"), ("k", "kw"))]
            close(s["qr"][live], y[0][0][live], 20 * 2.0 ** -24 * y[0][1][live])
            assert (s["qr"][3] == 0).all()
            for new, c, e in ((y[1][0], "kc", "ks"), (f64(s["v"]), "vc", "vs")):
                codes, scales = old[c].cpu().numpy(), old[e].cpu().numpy()
                for b in live:
                    page, row = serving.place(table, len(codes), d.P, b, int(pn[b]))
                    codes[page, :, row], scales[page, :, row] = ms.mx_pack(new[b].astype(np.float32))
                np.testing.assert_array_equal(s[c].cpu().numpy(), codes)
                np.testing.assert_array_equal(s[e].cpu().numpy(), scales)
            kv = [ms.mx_values(s[c].cpu().numpy(), s[e].cpu().numpy()) for c, e in (("kc", "ks"), ("vc", "vs"))]
            o, lse, tol, tol_lse = serving.attn_paged(f64(s["qr"]), *kv, table, (pos + 1).tolist(), d.D ** -0.5)
            close(s["o"], o, tol[:, :, None] + 2.0 ** -15 * np.abs(np.nan_to_num(kv[1])).max())
            assert (np.abs(f64(s["lse"])[live] - lse[live]) <= tol_lse[live]).all() and (f64(s["lse"])[3] == -np.inf).all()
            close(s["mid"], *product(f64(s["o"]).reshape(5, -1), lay["wo"], residual=f64(s["x"])))
            close(s["h"], *product(f64(s["mid"]), lay["w1"], f64(lay["b1"]), "silu"))
            close(s["out"], *product(f64(s["h"]), lay["w2"], residual=f64(s["mid"])))
        close(logits, *product(f64(seen[-1]["out"]), d.head))
        for b in range(5):
            args = [wish[n][b].item() for n in ("u", "temperature", "top_k", "top_p", "min_p")]
            want, lps = ms.sample(f64(logits)[b], *args, error=d.V * 2.0 ** -43)
            assert int(token[b]) in want
            lp = lps[want.index(int(token[b]))]
            assert abs(float(logp[b]) - lp) <= 260 * 2.0 ** -24 + 2.0 ** -24 * abs(lp)
        tokens = token


def test_captured_step_replays(ta):
    """A step captured once makes every later one, its own token fed back to it."""
    d = Decoder(ta)
    held = [3, 30, 0, 0, 64]
    d.prefill(held)
    eager = d.clone()
    tokens, pos = torch.zeros(5, dtype=I32, device="cuda"), torch.full((5,), -1, dtype=I32, device="cuda")
    lens, wish = torch.zeros(5, dtype=I32, device="cuda"), d.wish(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        d.step(tokens, None, pos, lens, wish)        # (nothing is appended at position -1)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logits, token, logp = d.step(tokens, None, pos, lens, wish)
    for step in range(6):
        at = torch.tensor([n + step if b != 3 else step // 2 if step % 2 else -1 for b, n in enumerate(held)],
                          dtype=I32, device="cuda")     # (slot 3 is idle every other step)
        pos.copy_(at), lens.copy_(at + 1)
        for n, t in d.wish(step).items():
            wish[n].copy_(t.roll(step) if n != "u" else t)
        before = tokens.clone()
        graph.replay()
        torch.cuda.synchronize()
        want = eager.step(before, None, at, at + 1, {n: t.clone() for n, t in wish.items()})
        for got, w in zip((logits, token, logp), want):
            assert torch.equal(got, w)
        for a, b in zip(d.layers, eager.layers):
            assert all(torch.equal(a[n], b[n]) for n in ("kc", "vc", "ks", "vs"))
        tokens.copy_(token)


def test_two_streams_at_once(ta):
    """Two decoders' steps on streams of their own, launched in turn, against the same
    steps one after the other."""
    ds = [Decoder(ta, seed) for seed in (5, 6)]
    for d in ds:
        d.prefill([10, 20, 40, 1, 70])
    alone = [d.clone() for d in ds]
    streams = [torch.cuda.Stream() for _ in ds]
    tokens = torch.arange(5, device="cuda")
    got = [None, None]
    torch.cuda.synchronize()
    for step in range(4):
        pos = torch.tensor([10, 20, 40, 1, 70], dtype=I32, device="cuda") + step
        wish = ds[0].wish(step)
        torch.cuda.synchronize()
        for i, d in enumerate(ds):
            with torch.cuda.stream(streams[i]):
                got[i] = d.step(tokens, None, pos, pos + 1, wish, stream=streams[i])
        torch.cuda.synchronize()
        for i, d in enumerate(alone):
            for a, b in zip(got[i], d.step(tokens, None, pos, pos + 1, wish)):
                assert torch.equal(a, b)
