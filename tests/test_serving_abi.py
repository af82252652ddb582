"""Refusals of the serving step's calls, on the CPU: the C entry points with fake
addresses (every call must fail validation), and the binding's own checks."""
import os

import pytest

from paper_2504_17577_amd import tileattn as ta

no_gpu = pytest.mark.skipif(os.path.exists("/dev/kfd"),
                            reason="fake-pointer validation cases run only without a GPU")

K, V, SEQ, POS, KC, VC, KS, VS, TAB = (0x100000000 * i for i in range(1, 10))
APPEND = dict(K=K, V=V, k_stride=1024, v_stride=1024, seq=SEQ, pos=POS, KC=KC, VC=VC, e4m3=0, ks=None, vs=None,
              table=TAB, T=40, B=4, Hkv=8, D=128, num_pages=100, page=64, per=20, stream=None)
CACHE_BAD = [
    (dict(KC=0), 1), (dict(VC=0), 1), (dict(table=0), 1),
    (dict(B=0), 2), (dict(Hkv=0), 2), (dict(D=0), 2), (dict(num_pages=0), 2), (dict(page=0), 2), (dict(per=-1), 2),
    (dict(per=1 << 25), 2), (dict(page=1 << 30, per=2), 2), (dict(num_pages=(1 << 28) + 1), 2),
    (dict(D=96), 3), (dict(page=8), 3), (dict(page=48), 3), (dict(ks=KS), 3), (dict(vs=VS), 3),
    (dict(KC=KC + 8), 4), (dict(VC=VC + 2), 4), (dict(table=TAB + 2), 4), (dict(e4m3=1, ks=KS + 1), 4),
    (dict(e4m3=1, vs=VS + 2), 4),
]


@no_gpu
@pytest.mark.parametrize("change,status", CACHE_BAD + [
    (dict(K=0), 1), (dict(V=0), 1), (dict(pos=0), 1),
    (dict(T=0), 2), (dict(T=-3), 2), (dict(seq=None, T=5), 2), (dict(k_stride=1016), 2), (dict(v_stride=1028), 2),
    (dict(k_stride=-1024), 2), (dict(k_stride=1 << 31), 2), (dict(T=2147483647), 2),
    (dict(K=K + 2), 4), (dict(V=V + 8), 4), (dict(seq=SEQ + 2), 4), (dict(pos=POS + 1), 4),
    (dict(VC=KC + 1024), 6), (dict(K=KC + 1024), 6), (dict(V=VC - 1024), 6), (dict(pos=VC + 16), 6),
    (dict(seq=KC), 6), (dict(table=KC + 100 * 64 * 8 * 128 * 2 - 4), 6), (dict(e4m3=1, ks=VC), 6),
], ids=str)
def test_append_refusals(change, status):
    a = dict(APPEND, **change)
    rc = ta.lib().kv_cache_append(*a.values())
    assert rc == status, f"{change}: got {ta.STATUS.get(rc, rc)}, want {ta.STATUS[status]}"


Q, LENS, O, LSE, WS = (0x100000000 * i for i in range(11, 16))
ATTN = dict(Q=Q, q_stride=4096, KC=KC, VC=VC, e4m3=0, ks=None, vs=None, table=TAB, lens=LENS, O=O, o_bf16=0, LSE=LSE,
            B=4, Hq=32, Hkv=8, D=128, num_pages=100, page=64, per=20, scale=0.1, parts=64, ws=WS,
            ws_bytes=1 << 20, stream=None)


@no_gpu
@pytest.mark.parametrize("change,status", CACHE_BAD + [
    (dict(Q=0), 1), (dict(lens=0), 1), (dict(O=0), 1), (dict(LSE=0), 1),
    (dict(Hq=0), 2), (dict(Hq=12), 2), (dict(q_stride=4088), 2), (dict(q_stride=4100), 2),
    (dict(Q=Q + 8), 4), (dict(O=O + 4), 4), (dict(LSE=LSE + 4), 4), (dict(lens=LENS + 2), 4),
    (dict(scale=-0.1), 5), (dict(scale=float("nan")), 5), (dict(scale=float("inf")), 5),
    (dict(O=Q + 4096), 6), (dict(O=KC), 6), (dict(LSE=VC + 64), 6), (dict(LSE=O + 16), 6), (dict(O=TAB - 16), 6),
    (dict(LSE=LENS - 16), 6), (dict(e4m3=1, ks=O), 6),
    (dict(parts=-1), 2), (dict(parts=4097), 2), (dict(B=1 << 19, per=1 << 20), 2), (dict(Hq=1 << 17), 2),
    (dict(ws=0), 8), (dict(ws_bytes=64 * 2 * 4 * 130 * 4 - 1), 8), (dict(ws=WS + 8), 4),
    (dict(ws=KC + 4096), 6), (dict(ws=O), 6), (dict(ws=LSE - 4096), 6), (dict(ws=TAB), 6),
], ids=str)
def test_attention_refusals(change, status):
    a = dict(ATTN, **change)
    rc = ta.lib().attn_decode_paged(*a.values())
    assert rc == status, f"{change}: got {ta.STATUS.get(rc, rc)}, want {ta.STATUS[status]}"


def test_paged_workspace_and_plan():
    assert ta.attn_paged_workspace_bytes(32, 8, 128, 64) == 64 * 2 * 4 * 130 * 4
    assert ta.attn_paged_workspace_bytes(5, 1, 64, 3) == 3 * 2 * 8 * 66 * 4       # rows in fours
    assert ta.attn_paged_workspace_bytes(48, 1, 64, 1) == 2 * 24 * 66 * 4         # two row blocks of 24
    assert ta.attn_paged_workspace_bytes(32, 8, 128, 0) == 0
    for bad in [(32, 5, 128, 4), (0, 1, 64, 4), (32, 8, 96, 4), (32, 8, 128, -1), (32, 8, 128, 4097)]:
        with pytest.raises(ta.TileAttnError):
            ta.attn_paged_workspace_bytes(*bad)
    for B in (1, 7, 64, 1000):
        for Hq, Hkv in ((1, 1), (32, 8), (64, 1)):
            for cap in (1, 100, 10000, 1 << 24):
                assert 0 <= ta.attn_paged_plan(B, Hq, Hkv, 128, 16, cap) <= 4096
    for bad in [(0, 1, 1, 64, 16, 1), (1, 3, 2, 64, 16, 1), (1, 1, 1, 32, 16, 1), (1, 1, 1, 64, 0, 1), (1, 1, 1, 64, 16, 0)]:
        with pytest.raises(ta.TileAttnError):
            ta.attn_paged_plan(*bad)


A, B, BIAS, R, C = (0x100000000 * i for i in range(1, 6))
GEMM = dict(A=A, B=B, bias=BIAS, R=R, C=C, c_bf16=0, act=1, M=40, N=64, K=1032, splits=2, ws=WS,
            ws_bytes=1 << 20, stream=None)


@no_gpu
@pytest.mark.parametrize("change,status", [
    (dict(A=0), 1), (dict(B=0), 1), (dict(C=0), 1),
    (dict(M=0), 2), (dict(N=0), 2), (dict(K=-8), 2), (dict(N=1 << 24), 2), (dict(K=1 << 22), 2),
    (dict(M=1 << 20, N=1 << 15), 2), (dict(M=1 << 20, K=1 << 20), 2), (dict(M=(1 << 20) + 1), 2), (dict(N=1 << 22, K=1 << 18), 2),
    (dict(splits=0), 2), (dict(splits=65), 2),
    (dict(N=60), 3), (dict(K=132), 3), (dict(act=-1), 3), (dict(act=5), 3),
    (dict(A=A + 8), 4), (dict(B=B + 2), 4), (dict(C=C + 4), 4), (dict(bias=BIAS + 8), 4), (dict(R=R + 4), 4),
    (dict(C=A + 16), 6), (dict(C=B + 16), 6), (dict(C=BIAS), 6), (dict(R=C + 16), 6), (dict(R=C - 16), 6),
    (dict(ws=0), 8), (dict(ws_bytes=2 * 2 * 40 * 128 * 4 - 1), 8), (dict(ws=WS + 8), 4), (dict(ws=A), 6), (dict(ws=B + 1024), 6),
    (dict(ws=C - 16), 6), (dict(ws=R), 6), (dict(ws=BIAS), 6),
], ids=str)
def test_gemm_refusals(change, status):
    a = dict(GEMM, **change)
    rc = ta.lib().gemm_bf16_epilogue(*a.values())
    assert rc == status, f"{change}: got {ta.STATUS.get(rc, rc)}, want {ta.STATUS[status]}"


def test_gemm_workspace_and_plan():
    assert ta.gemm_epilogue_workspace_bytes(40, 64, 512, 1) == 0
    assert ta.gemm_epilogue_workspace_bytes(40, 64, 512, 2) == 2 * 2 * 40 * 128 * 4  # two records of a strip's columns each
    assert ta.gemm_epilogue_workspace_bytes(40, 64, 512, 3) == 2 * 2 * 40 * 128 * 4  # 16 steps for 8 waves: two workgroups
    assert ta.gemm_epilogue_workspace_bytes(40, 64, 128, 3) == 0                     # four steps: one
    assert ta.gemm_epilogue_workspace_bytes(8, 14336, 4096, 3) == 256 * 2 * 8 * 128 * 4   # 112 x 3, in whole rounds
    assert ta.gemm_epilogue_plan(24, 14336, 4096) == 2 and ta.gemm_epilogue_plan(8, 40000, 4096) == 2
    assert ta.gemm_epilogue_plan(64, 28672, 8192) == 1 and ta.gemm_epilogue_plan(1, 4096, 64) == 1
    assert ta.gemm_epilogue_workspace_bytes(100, 64, 512, 3) == 3 * 100 * 64 * 4
    assert ta.gemm_epilogue_workspace_bytes(100, 64, 512, 30) == 8 * 100 * 64 * 4    # eight steps of 64
    assert ta.gemm_epilogue_workspace_bytes(4096, 8192, 8192, 2) == 0                # whole rounds of large tiles
    assert ta.gemm_epilogue_workspace_bytes(4000, 8200, 8200, 4) == 4 * 4000 * 8 * 4
    for M in (1, 16, 40, 65, 300, 4096):
        for N in (8, 64, 1000, 4096, 65536):
            for K in (8, 64, 1000, 4096, 65536):
                assert 1 <= ta.gemm_epilogue_plan(M, N, K) <= 64
    for bad in [(0, 8, 8), (1, 0, 8), (1, 8, -8), (1, 12, 8), (1, 8, 4), (1, 1 << 24, 8)]:
        with pytest.raises(ta.TileAttnError):
            ta.gemm_epilogue_plan(*bad)
    for bad in [(0, 8, 8, 2), (1, 0, 8, 2), (1, 8, 0, 2), (1, 8, 12, 2), (1, 8, 8, 0), (1, 8, 8, 65)]:
        with pytest.raises(ta.TileAttnError):
            ta.gemm_epilogue_workspace_bytes(*bad)


torch = pytest.importorskip("torch")


@pytest.fixture
def gpu_like(monkeypatch):
    """CPU tensors taken for GPU ones, so that only the binding's checks are left."""
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)


def cache_args(e4m3=False):
    dt = torch.float8_e4m3fn if e4m3 else torch.bfloat16
    kc, vc = (torch.zeros(6, 2, 16, 64, dtype=torch.uint8 if e4m3 else dt).view(dt) for _ in range(2))
    return dict(k_cache=kc, v_cache=vc, page_table=torch.zeros(3, 2, dtype=torch.int32))


SCALE = torch.ones(2)
BAD_CACHE_TENSORS = [
    dict(k_cache=torch.zeros(6, 2, 16, 64)), dict(v_cache=torch.zeros(6, 2, 16, 64)),
    dict(v_cache=torch.zeros(6, 2, 32, 64, dtype=torch.bfloat16)), dict(k_cache=torch.zeros(6, 2, 16, dtype=torch.bfloat16)),
    dict(v_cache=torch.zeros(6, 16, 2, 64, dtype=torch.bfloat16).transpose(1, 2)),
    dict(page_table=torch.zeros(3, 2, dtype=torch.int64)), dict(page_table=torch.zeros(6, dtype=torch.int32)),
    dict(page_table=torch.zeros(2, 3, dtype=torch.int32).t()), dict(k_scale=SCALE), dict(v_scale=SCALE),
]


@pytest.mark.parametrize("change", BAD_CACHE_TENSORS + [
    dict(k=torch.zeros(3, 2, 64)), dict(v=torch.zeros(2, 2, 64, dtype=torch.bfloat16)),
    dict(k=torch.zeros(3, 64, 2, dtype=torch.bfloat16).transpose(1, 2)),
    dict(k=torch.zeros(3, 4, 64, dtype=torch.bfloat16)[:, ::2]),
    dict(pos=torch.zeros(3)), dict(pos=torch.zeros(4, dtype=torch.int32)), dict(seq=torch.zeros(2, dtype=torch.int32)),
], ids=lambda c: "-".join(f"{n}{tuple(t.shape)}{t.dtype}" for n, t in c.items()))
def test_append_checks(gpu_like, change):
    kv = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    a = dict(k=kv, v=kv, **cache_args(), pos=torch.zeros(3, dtype=torch.int32))
    with pytest.raises((TypeError, ta.TileAttnError)):
        ta.kv_cache_append(**dict(a, **change))


@pytest.mark.parametrize("change", BAD_CACHE_TENSORS + [
    dict(q=torch.zeros(3, 4, 64)), dict(q=torch.zeros(2, 4, 64, dtype=torch.bfloat16)),
    dict(q=torch.zeros(3, 256, dtype=torch.bfloat16)), dict(q=torch.zeros(3, 4, 128, dtype=torch.bfloat16)),
    dict(q=torch.zeros(3, 4, 128, dtype=torch.bfloat16)[:, :, ::2]), dict(seq_lens=torch.zeros(3, dtype=torch.int64)),
    dict(out=torch.zeros(3, 4, 64, dtype=torch.bfloat16)), dict(lse=torch.zeros(3, 4, 1)),
], ids=lambda c: "-".join(f"{n}{tuple(t.shape)}{t.dtype}" for n, t in c.items()))
def test_attention_checks(gpu_like, change):
    a = dict(q=torch.zeros(3, 4, 64, dtype=torch.bfloat16), **cache_args(), seq_lens=torch.zeros(3, dtype=torch.int32))
    with pytest.raises((TypeError, ta.TileAttnError)):
        ta.attn_decode_paged(**dict(a, **change))
    with pytest.raises(TypeError):
        ta.attn_decode_paged(**a, out_dtype=torch.float16)


@pytest.mark.parametrize("change", [
    dict(a=torch.zeros(4, 16)), dict(b=torch.zeros(24, 16, dtype=torch.bfloat16)),
    dict(b=torch.zeros(24, 16, dtype=torch.bfloat16).t()), dict(bias=torch.zeros(24)),
    dict(bias=torch.zeros(16, dtype=torch.bfloat16)), dict(residual=torch.zeros(4, 24, dtype=torch.bfloat16)),
    dict(residual=torch.zeros(24)), dict(out=torch.zeros(4, 16)), dict(activation="tanh"), dict(out_dtype=torch.float16),
], ids=str)
def test_gemm_checks(gpu_like, change):
    a = dict(a=torch.zeros(4, 16, dtype=torch.bfloat16), b=torch.zeros(16, 24, dtype=torch.bfloat16))
    with pytest.raises((TypeError, ta.TileAttnError)):
        ta.gemm_bf16_epilogue(**dict(a, **change))
