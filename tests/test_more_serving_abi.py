"""Refusals of the serving step's calls on 4-bit numbers, on the CPU: the C entry
points with fake addresses (every call must fail validation), and the binding's own
checks."""
import os

import pytest

from paper_2504_17577_amd import tileattn as ta
from test_serving_abi import gpu_like  # noqa: F401

no_gpu = pytest.mark.skipif(os.path.exists("/dev/kfd"),
                            reason="fake-pointer validation cases run only without a GPU")

Q, K, V, QW, KW, CS, SEQ, POS, QO, KC, VC, KS, VS, TAB = (0x100000000 * i for i in range(1, 15))
ROPE = dict(Q=Q, K=K, V=V, q_stride=4096, k_stride=1024, v_stride=1024, qw=QW, kw=KW, eps=1e-6, cs=CS, positions=4096,
            rot=128, inter=0, seq=SEQ, pos=POS, QO=QO, KC=KC, VC=VC, type=2, ks=KS, vs=VS, table=TAB, T=40, B=4, Hq=32,
            Hkv=8, D=128, num_pages=100, page=64, per=20, stream=None)
CACHE_BAD = [
    (dict(KC=0), 1), (dict(VC=0), 1), (dict(table=0), 1), (dict(ks=0), 1), (dict(vs=0), 1),
    (dict(B=0), 2), (dict(Hkv=0), 2), (dict(D=0), 2), (dict(num_pages=0), 2), (dict(page=0), 2), (dict(per=-1), 2),
    (dict(per=1 << 25), 2), (dict(page=1 << 30, per=2), 2), (dict(num_pages=(1 << 28) + 1), 2),
    (dict(D=96), 3), (dict(page=8), 3), (dict(page=48), 3),
    (dict(KC=KC + 8), 4), (dict(VC=VC + 2), 4), (dict(table=TAB + 2), 4), (dict(ks=KS + 8), 4), (dict(vs=VS + 4), 4),
]


@no_gpu
@pytest.mark.parametrize("change,status", CACHE_BAD + [
    (dict(Q=0), 1), (dict(K=0), 1), (dict(V=0), 1), (dict(pos=0), 1), (dict(QO=0), 1),
    (dict(T=0), 2), (dict(T=1 << 24), 2), (dict(seq=None, T=5), 2), (dict(Hq=-1), 2), (dict(Hq=(1 << 16) + 1), 2),
    (dict(q_stride=4088), 2), (dict(q_stride=4100), 2), (dict(k_stride=1016), 2), (dict(v_stride=1028), 2),
    (dict(q_stride=1 << 31), 2), (dict(k_stride=1 << 31), 2), (dict(v_stride=-1024), 2),
    (dict(positions=0), 2), (dict(positions=-5), 2), (dict(cs=None, rot=0), 2),
    (dict(type=3), 3), (dict(type=-1), 3), (dict(type=0), 3), (dict(rot=8), 3), (dict(rot=0), 3), (dict(rot=144), 3),
    (dict(rot=-16), 3), (dict(rot=40), 3), (dict(cs=None, positions=0), 3),
    (dict(eps=-1e-6), 5), (dict(eps=float("nan")), 5), (dict(eps=float("inf")), 5),
    (dict(Q=Q + 2), 4), (dict(K=K + 8), 4), (dict(V=V + 2), 4), (dict(QO=QO + 8), 4), (dict(qw=QW + 2), 4),
    (dict(kw=KW + 8), 4), (dict(cs=CS + 4), 4), (dict(seq=SEQ + 2), 4), (dict(pos=POS + 1), 4),
    (dict(type=1, ks=KS + 2), 4), (dict(type=1, vs=VS + 1), 4),
    (dict(QO=Q), 6), (dict(QO=KC + 16), 6), (dict(VC=KC + 1024), 6), (dict(KC=KS - 16), 6), (dict(vs=KS + 1024), 6),
    (dict(ks=VC), 6), (dict(ks=POS), 6), (dict(vs=TAB), 6), (dict(QO=CS + 4096 * 128 * 4 - 16), 6), (dict(KC=QW), 6),
    (dict(VC=KW), 6), (dict(QO=SEQ), 6), (dict(KC=V + 1024), 6), (dict(type=1, ks=VC), 6), (dict(QO=K), 6),
], ids=str)
def test_rope_refusals(change, status):
    a = dict(ROPE, **change)
    rc = ta.lib().qk_norm_rope_append(*a.values())
    assert rc == status, f"{change}: got {ta.STATUS.get(rc, rc)}, want {ta.STATUS[status]}"


LENS, O, LSE, WS = (0x100000000 * i for i in range(15, 19))
ATTN = dict(Q=Q, q_stride=4096, KC=KC, VC=VC, ks=KS, vs=VS, table=TAB, lens=LENS, O=O, o_bf16=0, LSE=LSE,
            B=4, Hq=32, Hkv=8, D=128, num_pages=100, page=64, per=20, scale=0.1, parts=64, ws=WS,
            ws_bytes=1 << 20, stream=None)


@no_gpu
@pytest.mark.parametrize("change,status", CACHE_BAD + [
    (dict(Q=0), 1), (dict(lens=0), 1), (dict(O=0), 1), (dict(LSE=0), 1), (dict(Hq=12), 2), (dict(q_stride=4088), 2),
    (dict(Q=Q + 8), 4), (dict(O=O + 4), 4), (dict(LSE=LSE + 4), 4), (dict(lens=LENS + 2), 4), (dict(scale=-0.1), 5),
    (dict(scale=float("nan")), 5), (dict(O=Q + 4096), 6), (dict(O=KC), 6), (dict(LSE=VC + 64), 6), (dict(O=KS + 16), 6),
    (dict(LSE=VS + 100 * 64 * 8 * 4 - 16), 6), (dict(O=KC + 100 * 64 * 8 * 64 - 16), 6), (dict(LSE=O + 16), 6),
    (dict(parts=-1), 2), (dict(parts=4097), 2), (dict(ws=0), 8), (dict(ws_bytes=64 * 2 * 4 * 130 * 4 - 1), 8),
    (dict(ws=WS + 8), 4), (dict(ws=KS + 4096), 6), (dict(ws=VS), 6), (dict(ws=O), 6),
], ids=str)
def test_attention_refusals(change, status):
    a = dict(ATTN, **change)
    rc = ta.lib().attn_decode_paged_mxfp4(*a.values())
    assert rc == status, f"{change}: got {ta.STATUS.get(rc, rc)}, want {ta.STATUS[status]}"


A, W, S, BIAS, R, C = (0x100000000 * i for i in range(1, 7))
GEMM = dict(A=A, W=W, S=S, bias=BIAS, R=R, C=C, c_bf16=0, act=1, M=40, N=64, K=4128, parts=2, ws=WS,
            ws_bytes=1 << 20, stream=None)


@no_gpu
@pytest.mark.parametrize("change,status", [
    (dict(A=0), 1), (dict(W=0), 1), (dict(S=0), 1), (dict(C=0), 1),
    (dict(M=0), 2), (dict(N=0), 2), (dict(K=-32), 2), (dict(N=1 << 24), 2), (dict(K=1 << 22), 2),
    (dict(M=1 << 20, N=1 << 15), 2), (dict(M=1 << 20, K=1 << 20), 2), (dict(M=(1 << 20) + 1), 2), (dict(N=1 << 22, K=1 << 18), 2),
    (dict(parts=-1), 2), (dict(parts=4097), 2), (dict(N=60), 3), (dict(K=4112), 3), (dict(act=-1), 3), (dict(act=5), 3),
    (dict(A=A + 8), 4), (dict(W=W + 2), 4), (dict(C=C + 4), 4), (dict(bias=BIAS + 8), 4), (dict(R=R + 4), 4),
    (dict(C=A + 16), 6), (dict(C=W + 16), 6), (dict(C=S), 6), (dict(S=C + 64 * 40 * 4 - 1), 6), (dict(C=BIAS), 6),
    (dict(R=C + 16), 6), (dict(R=C - 16), 6),
    (dict(ws=0), 8), (dict(ws_bytes=2 * 2 * 40 * 64 * 4 - 1), 8), (dict(ws=WS + 8), 4), (dict(ws=A), 6), (dict(ws=W + 1024), 6),
    (dict(ws=S + 16), 6), (dict(ws=C - 16), 6), (dict(ws=R), 6), (dict(ws=BIAS), 6),
], ids=str)
def test_gemm_refusals(change, status):
    a = dict(GEMM, **change)
    rc = ta.lib().gemm_mxfp4_epilogue(*a.values())
    assert rc == status, f"{change}: got {ta.STATUS.get(rc, rc)}, want {ta.STATUS[status]}"


def test_gemm_plan():
    for M in (1, 16, 40, 65, 300, 4096):
        for N in (8, 64, 1000, 4096, 65536):
            for K in (32, 64, 992, 4096, 65536):
                n = ta.gemm_mxfp4_plan(M, N, K)
                assert 0 <= n <= 256 and ta.gemm_mxfp4_workspace_bytes(M, N, K, 0) == 0
                assert (ta.gemm_mxfp4_workspace_bytes(M, N, K, n) > 0) == (n > 0)
    assert ta.gemm_mxfp4_workspace_bytes(40, 64, 4128, 2) == 2 * 2 * 40 * 64 * 4        # two records of a strip each
    assert ta.gemm_mxfp4_workspace_bytes(40, 64, 256, 30) == 2 * 2 * 40 * 64 * 4        # two steps
    assert ta.gemm_mxfp4_workspace_bytes(3, 64, 4096, 30) == 16 * 2 * 3 * 16 * 4        # 128 steps, eight waves
    assert ta.gemm_mxfp4_workspace_bytes(100, 256, 1024, 9) == 9 * 2 * 128 * 128 * 4    # tiles
    assert ta.gemm_mxfp4_workspace_bytes(1 << 20, 1 << 14, (1 << 20) - 32, 9) == 0             # steps past 32 bits: whole tiles
    for bad in [(0, 8, 32), (1, 0, 32), (1, 8, -32), (1, 12, 32), (1, 8, 48), (1, 1 << 24, 32)]:
        with pytest.raises(ta.TileAttnError):
            ta.gemm_mxfp4_plan(*bad)
        with pytest.raises(ta.TileAttnError):
            ta.gemm_mxfp4_workspace_bytes(*bad, 2)
    for parts in (-1, 4097):
        with pytest.raises(ta.TileAttnError):
            ta.gemm_mxfp4_workspace_bytes(1, 8, 32, parts)


L, U, TEMP, TOPK, TOPP, MINP, TOKEN, LOGP = (0x100000000 * i for i in range(1, 9))
SAMPLE = dict(L=L, stride=50000, bf16=1, u=U, T=TEMP, k=TOPK, p=TOPP, m=MINP, token=TOKEN, logp=LOGP, B=3, V=50000, ws=WS,
              ws_bytes=1 << 24, stream=None)
SAMPLE_WS = ta.sample_workspace_bytes(3, 50000)


@no_gpu
@pytest.mark.parametrize("change,status", [
    (dict(L=0), 1), (dict(u=0), 1), (dict(token=0), 1), (dict(logp=0), 1),
    (dict(B=0), 2), (dict(V=0), 2), (dict(B=(1 << 16) + 1), 2), (dict(V=(1 << 20) + 1), 2), (dict(V=-1), 2),
    (dict(stride=-1), 2), (dict(stride=(1 << 30) + 1), 2), (dict(stride=-50000), 2),
    (dict(L=L + 1), 4), (dict(L=L + 2, bf16=0), 4), (dict(u=U + 2), 4), (dict(T=TEMP + 1), 4), (dict(k=TOPK + 2), 4),
    (dict(p=TOPP + 2), 4), (dict(m=MINP + 3), 4), (dict(token=TOKEN + 2), 4), (dict(logp=LOGP + 1), 4),
    (dict(token=LOGP + 4), 6), (dict(token=L), 6), (dict(logp=L + 2 * 149996), 6), (dict(logp=U), 6), (dict(token=TEMP), 6),
    (dict(logp=TOPK - 4), 6), (dict(token=TOPP + 8), 6), (dict(logp=MINP), 6),
    (dict(ws=0), 8), (dict(ws_bytes=SAMPLE_WS - 1), 8), (dict(ws=WS + 8), 4), (dict(ws=L - 16), 6), (dict(ws=TOKEN), 6),
    (dict(ws=LOGP - 1024), 6), (dict(ws=U - 64), 6), (dict(ws=TOPK), 6),
], ids=str)
def test_sample_refusals(change, status):
    a = dict(SAMPLE, **change)
    rc = ta.lib().sample_logits(*a.values())
    assert rc == status, f"{change}: got {ta.STATUS.get(rc, rc)}, want {ta.STATUS[status]}"


def test_sample_workspace():
    assert ta.sample_workspace_bytes(1, 1) == 0 and 0 < SAMPLE_WS < 1 << 20
    for bad in [(0, 10), (10, 0), ((1 << 16) + 1, 10), (10, (1 << 20) + 1)]:
        with pytest.raises(ta.TileAttnError):
            ta.sample_workspace_bytes(*bad)


torch = pytest.importorskip("torch")
BF16, U8, I32 = torch.bfloat16, torch.uint8, torch.int32


def cache_args():
    return dict(k_cache=torch.zeros(6, 2, 16, 32, dtype=U8), v_cache=torch.zeros(6, 2, 16, 32, dtype=U8),
                k_scale=torch.zeros(6, 2, 16, 2, dtype=U8), v_scale=torch.zeros(6, 2, 16, 2, dtype=U8),
                page_table=torch.zeros(3, 2, dtype=I32))


BAD_CACHE_TENSORS = [
    dict(k_scale=None), dict(v_scale=None), dict(k_scale=torch.ones(2)), dict(v_scale=torch.zeros(6, 2, 16, 2)),
    dict(k_scale=torch.zeros(6, 2, 16, 1, dtype=U8)), dict(v_scale=torch.zeros(6, 2, 2, 16, dtype=U8).transpose(2, 3)),
    dict(v_cache=torch.zeros(6, 2, 16, 64, dtype=BF16)), dict(v_cache=torch.zeros(6, 2, 16, 64, dtype=U8)),
    dict(k_cache=torch.zeros(6, 2, 16, 32, dtype=torch.int8)), dict(k_cache=torch.zeros(6, 2, 16, dtype=U8)),
    dict(k_cache=torch.zeros(6, 2, 16, 64, dtype=BF16), v_cache=torch.zeros(6, 2, 16, 64, dtype=BF16)),
]
describe = lambda c: "-".join(f"{n}{tuple(t.shape)}{t.dtype}" if t is not None else n for n, t in c.items())  # noqa: E731


@pytest.mark.parametrize("change", BAD_CACHE_TENSORS + [
    dict(q=torch.zeros(3, 4, 64)), dict(q=torch.zeros(2, 4, 64, dtype=BF16)), dict(q=torch.zeros(3, 256, dtype=BF16)),
    dict(k=torch.zeros(3, 64, 2, dtype=BF16).transpose(1, 2)), dict(v=torch.zeros(3, 2, 128, dtype=BF16)),
    dict(pos=torch.zeros(3)), dict(seq=torch.zeros(2, dtype=I32)), dict(q_weight=torch.zeros(64)),
    dict(k_weight=torch.zeros(32, dtype=BF16)), dict(cos_sin=torch.zeros(10, 64, dtype=BF16)), dict(cos_sin=torch.zeros(64)),
    dict(cos_sin=torch.zeros(64, 10).t()), dict(out=torch.zeros(3, 4, 64)), dict(out=torch.zeros(3, 5, 64, dtype=BF16)),
], ids=describe)
def test_rope_checks(gpu_like, change):  # noqa: F811
    kv = torch.zeros(3, 2, 64, dtype=BF16)
    a = dict(q=torch.zeros(3, 4, 64, dtype=BF16), k=kv, v=kv, **cache_args(), pos=torch.zeros(3, dtype=I32))
    with pytest.raises((TypeError, ta.TileAttnError)):
        ta.qk_norm_rope_append(**dict(a, **change))


@pytest.mark.parametrize("change", BAD_CACHE_TENSORS, ids=describe)
def test_append_and_attention_checks(gpu_like, change):  # noqa: F811
    kv = torch.zeros(3, 2, 64, dtype=BF16)
    with pytest.raises((TypeError, ta.TileAttnError)):
        ta.kv_cache_append(**dict(dict(k=kv, v=kv, **cache_args(), pos=torch.zeros(3, dtype=I32)), **change))
    with pytest.raises((TypeError, ta.TileAttnError)):
        ta.attn_decode_paged(**dict(dict(q=torch.zeros(3, 4, 64, dtype=BF16), **cache_args(), seq_lens=torch.zeros(3, dtype=I32)), **change))


@pytest.mark.parametrize("change", [
    dict(a=torch.zeros(4, 64)), dict(a=torch.zeros(4, 48, dtype=BF16)), dict(a=torch.zeros(64, 4, dtype=BF16).t()),
    dict(w=torch.zeros(24, 32)), dict(w=torch.zeros(24, 31, dtype=U8)), dict(w=torch.zeros(32, 24, dtype=U8).t()),
    dict(w=torch.zeros(24 * 32, dtype=U8)), dict(w_scale=torch.zeros(24, 2)), dict(w_scale=torch.zeros(24, 1, dtype=U8)),
    dict(w=torch.zeros(20, 32, dtype=U8), w_scale=torch.zeros(20, 2, dtype=U8)), dict(bias=torch.zeros(24)),
    dict(bias=torch.zeros(16, dtype=BF16)), dict(residual=torch.zeros(4, 24, dtype=BF16)),
    dict(out=torch.zeros(4, 16)), dict(activation="tanh"), dict(out_dtype=torch.float16),
], ids=str)
def test_gemm_checks(gpu_like, change):  # noqa: F811
    a = dict(a=torch.zeros(4, 64, dtype=BF16), w=torch.zeros(24, 32, dtype=U8), w_scale=torch.zeros(24, 2, dtype=U8))
    with pytest.raises((TypeError, ta.TileAttnError)):
        ta.gemm_mxfp4_epilogue(**dict(a, **change))


@pytest.mark.parametrize("change", [
    dict(logits=torch.zeros(3, 40, dtype=torch.float16)), dict(logits=torch.zeros(40)), dict(logits=torch.zeros(40, 3).t()),
    dict(logits=torch.zeros(3, 80)[:, ::2]), dict(u=torch.zeros(2)), dict(u=torch.zeros(3, dtype=torch.float64)),
    dict(temperature=torch.zeros(1)), dict(top_k=torch.zeros(3)), dict(top_k=torch.zeros(3, dtype=torch.int64)),
    dict(top_p=torch.zeros(3, 1)), dict(min_p=torch.zeros(6)[::2]), dict(token=torch.zeros(3)),
    dict(logp=torch.zeros(3, dtype=BF16)), dict(workspace=torch.zeros(100)),
], ids=describe)
def test_sample_checks(gpu_like, change):  # noqa: F811
    a = dict(logits=torch.zeros(3, 40), u=torch.zeros(3))
    with pytest.raises((TypeError, ta.TileAttnError)):
        ta.sample_logits(**dict(a, **change))
