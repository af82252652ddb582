"""The serving calls together, as a decoder's step uses them: a fused projection
with bias, its K and V appended to the paged cache, attention over the cache, the
output projection onto the residual stream in place, and an MLP.  Every call of
the step is held to the oracle on the inputs that it got; a captured step,
replayed, to the same step run eagerly, bit for bit; and the calls on side
streams, with shared workspaces and after one another to themselves."""
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


def f64(t):
    return t.double().cpu().numpy()


class Decoder:
    """Two layers of a grouped-query decoder with a batch of five slots."""
    HID, HQ, HKV, D, FF, B, P, PER = 264, 6, 2, 64, 520, 5, 16, 6

    def __init__(self, ta, e4m3, seed=0):
        self.ta, g = ta, torch.Generator(device="cuda").manual_seed(seed)
        n = lambda *s, std=1.0: (torch.randn(*s, generator=g, device="cuda") * std).to(BF16)   # noqa: E731
        qkv = (self.HQ + 2 * self.HKV) * self.D
        self.layers = [dict(wqkv=n(self.HID, qkv, std=self.HID ** -0.5), bqkv=n(qkv, std=0.3),
                            wo=n(self.HQ * self.D, self.HID, std=0.05), w1=n(self.HID, self.FF, std=0.06),
                            b1=n(self.FF, std=0.3), w2=n(self.FF, self.HID, std=0.04)) for _ in range(2)]
        pages = self.B * self.PER + 3
        self.table = torch.randperm(pages, generator=g, device="cuda")[:self.B * self.PER].to(I32).view(self.B, self.PER)
        dt = E4M3 if e4m3 else BF16
        shape = (pages, self.HKV, self.P, self.D)
        for lay in self.layers:   # NaN wherever nothing has been written
            lay["kc"], lay["vc"] = (torch.full(shape, 0x7F, dtype=torch.uint8, device="cuda").view(E4M3) if e4m3
                                    else torch.full(shape, float("nan"), dtype=dt, device="cuda") for _ in range(2))
            lay["ks"], lay["vs"] = (torch.rand(2, self.HKV, generator=g, device="cuda") * 0.01 + 0.01).unbind(0) \
                if e4m3 else (None, None)

    def clone(self):
        other = object.__new__(Decoder)
        other.__dict__.update(self.__dict__)
        other.layers = [dict(lay, kc=lay["kc"].clone(), vc=lay["vc"].clone()) for lay in self.layers]
        return other

    def step(self, x, seq, pos, lens, seen=None):
        """One pass over the tokens x [T, HID] at positions pos of sequences seq (for one
        token per slot: seq None, and attention); x is the residual stream, updated."""
        T, ta = x.shape[0], self.ta
        for lay in self.layers:
            qkv = ta.gemm_bf16_epilogue(x, lay["wqkv"], bias=lay["bqkv"], out_dtype=BF16).view(T, -1, self.D)
            q, k, v = qkv[:, :self.HQ], qkv[:, self.HQ:self.HQ + self.HKV], qkv[:, self.HQ + self.HKV:]
            ta.kv_cache_append(k, v, lay["kc"], lay["vc"], self.table, pos, seq=seq, k_scale=lay["ks"], v_scale=lay["vs"])
            if seq is not None:
                continue   # a prefill's attention is not what is looked at here
            o, lse = ta.attn_decode_paged(q, lay["kc"], lay["vc"], self.table, lens, k_scale=lay["ks"],
                                          v_scale=lay["vs"], out_dtype=BF16)
            before = x.clone() if seen is not None else None
            ta.gemm_bf16_epilogue(o.view(T, -1), lay["wo"], residual=x, out=x, out_dtype=BF16)
            mid = x.clone() if seen is not None else None
            h = ta.gemm_bf16_epilogue(x, lay["w1"], bias=lay["b1"], activation="gelu_tanh", out_dtype=BF16)
            ta.gemm_bf16_epilogue(h, lay["w2"], residual=x, out=x, out_dtype=BF16)
            if seen is not None:
                seen.append(dict(lay=lay, q=q, k=k, v=v, o=o, lse=lse, x0=before, qkv=qkv.view(T, -1), x1=mid, h=h,
                                 x2=x.clone(), kc=lay["kc"].clone(), vc=lay["vc"].clone()))
        return x

    def prefill(self, lens, seed=1):
        """Fills the caches with lens[b] tokens of sequence b, in one ragged batch with padding rows."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        seq = torch.tensor([b for b, n in enumerate(lens) for _ in range(n)] + [0, 3], dtype=I32, device="cuda")
        pos = torch.tensor([t for n in lens for t in range(n)] + [-1, -1], dtype=I32, device="cuda")
        self.step(torch.randn(len(seq), self.HID, generator=g, device="cuda").to(BF16), seq, pos, None)


def close(got, want, tol):
    err = np.abs(f64(got) - want)
    assert (err <= tol + 2.0 ** -8 * np.abs(want)).all(), float((err / (tol + 2.0 ** -8 * np.abs(want))).max())


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_step_against_oracle(ta, e4m3):
    d = Decoder(ta, e4m3)
    held = [0, 15, 16, 0, 77]                       # slot 3 stays idle
    d.prefill(held)
    g = torch.Generator(device="cuda").manual_seed(2)
    for step in range(3):
        pos = torch.tensor([n + step if b != 3 else -1 for b, n in enumerate(held)], dtype=I32, device="cuda")
        before = [(lay["kc"].clone(), lay["vc"].clone()) for lay in d.layers]
        seen = []
        d.step(torch.randn(5, d.HID, generator=g, device="cuda").to(BF16), None, pos, pos + 1, seen)
        bits = lambda t: t.contiguous().view(torch.uint8 if t.dtype == E4M3 else torch.int16).cpu().numpy()  # noqa: E731
        for s, (kc0, vc0) in zip(seen, before):
            lay = s["lay"]
            close(s["qkv"], *serving.gemm_epilogue(f64(s["x0"]), f64(lay["wqkv"]), f64(lay["bqkv"])))
            for new, c0, c1, sc in ((s["k"], kc0, s["kc"], lay["ks"]), (s["v"], vc0, s["vc"], lay["vs"])):
                kind = np.uint8 if e4m3 else np.uint16
                want = serving.append(bits(new).view(np.uint16), bits(c0).view(kind), d.table.cpu().numpy(),
                                      pos.cpu().numpy(), None, None if sc is None else sc.cpu().numpy())
                np.testing.assert_array_equal(bits(c1).view(kind), want)
            sc = [None if t is None else f64(t) for t in (lay["ks"], lay["vs"])]
            o, lse, tol, tol_lse = serving.attn_paged(f64(s["q"]), f64(s["kc"]), f64(s["vc"]), d.table.cpu().numpy(),
                                                      (pos + 1).tolist(), d.D ** -0.5, *sc)
            top = np.nan_to_num(np.abs(f64(s["vc"]))).max() * (1 if sc[1] is None else sc[1].max())
            close(s["o"], o, tol[:, :, None] + 2.0 ** -15 * top)
            got = f64(s["lse"])
            assert (got[3] == -np.inf).all() and (f64(s["o"])[3] == 0).all()
            live = [0, 1, 2, 4]
            assert (np.abs(got[live] - lse[live]) <= tol_lse[live]).all()
            close(s["x1"], *serving.gemm_epilogue(f64(s["o"]).reshape(5, -1), f64(lay["wo"]), residual=f64(s["x0"])))
            close(s["h"], *serving.gemm_epilogue(f64(s["x1"]), f64(lay["w1"]), f64(lay["b1"]), "gelu_tanh"))
            close(s["x2"], *serving.gemm_epilogue(f64(s["h"]), f64(lay["w2"]), residual=f64(s["x1"])))


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_captured_step_replays(ta, e4m3):
    """A step captured once serves every later one: positions and lengths are read
    from the arrays at each replay, idle slots included."""
    d = Decoder(ta, e4m3)
    held = [3, 30, 0, 0, 64]
    d.prefill(held)
    eager = d.clone()
    x, pos = torch.zeros(5, d.HID, dtype=BF16, device="cuda"), torch.full((5,), -1, dtype=I32, device="cuda")
    lens = torch.zeros(5, dtype=I32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        d.step(x, None, pos, lens)                   # (nothing is appended at position -1)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d.step(x, None, pos, lens)
    g = torch.Generator(device="cuda").manual_seed(3)
    for step in range(5):
        new = torch.randn(5, d.HID, generator=g, device="cuda").to(BF16)
        at = torch.tensor([n + step if (b, step % 2) != (3, 0) and n + step < 96 else -1 for b, n in enumerate(held)],
                          dtype=I32, device="cuda")
        x.copy_(new), pos.copy_(at), lens.copy_(at + 1)
        graph.replay()
        want = eager.step(new.clone(), None, at, at + 1)
        torch.cuda.synchronize()
        # (slot 3's position 0 is never written: the NaN there is its own alone)
        assert torch.equal(x.view(torch.int16), want.view(torch.int16)), f"replay {step}"
        assert x[[0, 1, 2, 4]].isfinite().all()
        for a, b in zip(d.layers, eager.layers):
            for c in ("kc", "vc"):
                assert torch.equal(a[c].view(torch.uint8), b[c].view(torch.uint8)), f"replay {step} {c}"


def paged(B, Hkv, D, P, n, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    per = -(-n // P)
    kc, vc = (torch.randn(B * per, Hkv, P, D, generator=g, device="cuda").to(BF16) for _ in range(2))
    table = torch.randperm(B * per, generator=g, device="cuda").to(I32).view(B, per)
    return kc, vc, table, torch.randint(0, n + 1, (B,), generator=g, device="cuda").to(I32)


def test_two_graphs_share_a_workspace(ta):
    """Two captured calls of other sizes on one workspace, replayed in turn."""
    calls, graphs = [], []
    ws = torch.empty(ta.attn_paged_workspace_bytes(16, 2, 128, 64), dtype=torch.uint8, device="cuda")
    for seed, (B, Hq, D) in enumerate([(3, 16, 128), (7, 4, 64)]):
        kv = paged(B, 2, D, 32, 900, seed)
        q = torch.randn(B, Hq, D, device="cuda").to(BF16)
        out, lse = torch.empty(B, Hq, D, device="cuda"), torch.empty(B, Hq, device="cuda")
        calls.append(dict(q=q, k_cache=kv[0], v_cache=kv[1], page_table=kv[2], seq_lens=kv[3], num_parts=64, workspace=ws,
                          out=out, lse=lse))
    want = [[t.clone() for t in ta.attn_decode_paged(**dict(c, workspace=None, out=None, lse=None))] for c in calls]
    torch.cuda.synchronize()
    for c in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            ta.attn_decode_paged(**c)
    for turn in range(3):
        for i in (0, 1, 1, 0):
            calls[i]["out"].fill_(7), calls[i]["lse"].fill_(7)
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(calls[i]["out"], want[i][0]) and torch.equal(calls[i]["lse"], want[i][1]), (turn, i)


def test_calls_on_a_side_stream(ta):
    """With ``stream`` given the calls run there, in order with the stream's other work."""
    kc, vc, table, lens = paged(4, 2, 64, 16, 700)
    q = torch.randn(4, 8, 64, device="cuda").to(BF16)
    a, b = torch.randn(20, 1024, device="cuda").to(BF16), torch.randn(1024, 512, device="cuda").to(BF16)
    k = torch.randn(4, 2, 64, device="cuda").to(BF16)
    pos = lens.clamp(max=699)
    k2, v2 = kc.clone(), vc.clone()
    ta.kv_cache_append(k, k, k2, v2, table, pos)
    want = ta.attn_decode_paged(q, k2, v2, table, lens, num_parts=100), ta.gemm_bf16_epilogue(a, b, num_splits=8)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        kc2, vc2 = kc.clone(), vc.clone()
        o, lse, c = torch.empty(4, 8, 64, device="cuda"), torch.empty(4, 8, device="cuda"), torch.empty(20, 512, device="cuda")
        side.wait_stream(torch.cuda.current_stream())
        ta.kv_cache_append(k, k, kc2, vc2, table, pos, stream=side)
        ta.attn_decode_paged(q, kc2, vc2, table, lens, num_parts=100, out=o, lse=lse, stream=side)
        ta.gemm_bf16_epilogue(a, b, num_splits=8, out=c, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(kc2, k2) and torch.equal(o, want[0][0]) and torch.equal(lse, want[0][1]) and torch.equal(c, want[1])
        torch.cuda.synchronize()


def test_results_do_not_depend_on_timing(ta):
    kc, vc, table, lens = paged(9, 4, 128, 16, 3000)
    q = torch.randn(9, 16, 128, device="cuda").to(BF16)
    a, b = torch.randn(33, 4096, device="cuda").to(BF16), torch.randn(4096, 1000, device="cuda").to(BF16)
    c, d = torch.randn(130, 4096, device="cuda").to(BF16), torch.randn(4096, 1000, device="cuda").to(BF16)
    run = lambda: (*ta.attn_decode_paged(q, kc, vc, table, lens), ta.gemm_bf16_epilogue(a, b), ta.gemm_bf16_epilogue(c, d))  # noqa: E731
    first = run()
    for _ in range(5):
        for x, y in zip(run(), first):
            assert torch.equal(x, y)
