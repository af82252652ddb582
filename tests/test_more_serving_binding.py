"""The host logic of the serving step's calls on 4-bit numbers and of the next token's
choice on the CPU, with stand-ins for GPU tensors and streams and the C calls recorded
(test_binding.py's): workspaces come from the launch stream's pool, which C call a cache's
type takes, what is passed on."""
import pytest

torch = pytest.importorskip("torch")

from paper_2504_17577_amd import tileattn as ta  # noqa: E402
from test_binding import BF16, F32, FakeLib, FakeStream, fake  # noqa: E402, F401
from test_serving_binding import t  # noqa: E402

I32, U8 = torch.int32, torch.uint8


@pytest.fixture
def calls(fake, monkeypatch):  # noqa: F811
    monkeypatch.setattr(FakeLib, "LAUNCHES", FakeLib.LAUNCHES + (
        "kv_cache_append", "qk_norm_rope_append", "attn_decode_paged", "attn_decode_paged_mxfp4", "gemm_mxfp4_epilogue", "sample_logits"))
    return fake


def cache4(per=1000):
    return dict(k_cache=t(10, 2, 64, 64, dtype=U8), v_cache=t(10, 2, 64, 64, dtype=U8), page_table=t(3, per, dtype=I32),
                k_scale=t(10, 2, 64, 4, dtype=U8), v_scale=t(10, 2, 64, 4, dtype=U8))


def product(M, N, K, **kw):
    return ta.gemm_mxfp4_epilogue(t(M, K), t(N, K // 2, dtype=U8), t(N, K // 32, dtype=U8), out=t(M, N, dtype=F32), **kw)


@pytest.mark.parametrize("side", [True, False], ids=["side", "current"])
def test_workspaces_are_allocated_on_the_launch_stream(calls, side):
    s = FakeStream() if side else None
    ta.attn_decode_paged(t(3, 8, 128), seq_lens=t(3, dtype=I32), out=t(3, 8, 128, dtype=F32), lse=t(3, 8, dtype=F32), stream=s, **cache4())
    product(64, 4096, 4096, stream=s)
    ta.sample_logits(t(4, 100000), t(4, dtype=F32), token=t(4, dtype=I32), logp=t(4, dtype=F32), stream=s)
    assert [m.dtype for m in calls.made] == [U8] * 3 and all(m.stream is s for m in calls.made)
    parts = ta.attn_paged_mxfp4_plan(3, 8, 2, 128, 64, 1000)
    assert [m.numel() for m in calls.made] == [
        ta.attn_paged_workspace_bytes(8, 2, 128, parts),
        ta.gemm_mxfp4_workspace_bytes(64, 4096, 4096, ta.gemm_mxfp4_plan(64, 4096, 4096)), ta.sample_workspace_bytes(4, 100000)]
    assert [n for n, _ in calls.calls] == ["attn_decode_paged_mxfp4", "gemm_mxfp4_epilogue", "sample_logits"]
    assert [a[-1] for _, a in calls.calls] == [0x5000 if side else 0] * 3


def test_calls_that_need_no_workspace_allocate_none(calls):
    c = cache4(4)
    ta.attn_decode_paged(t(3, 8, 128), seq_lens=t(3, dtype=I32), out=t(3, 8, 128, dtype=F32), lse=t(3, 8, dtype=F32), **c)
    product(1, 4096, 4096)
    ta.sample_logits(t(4, 32000), t(4, dtype=F32), token=t(4, dtype=I32), logp=t(4, dtype=F32))
    kv, pos, out = t(3, 2, 128), t(3, dtype=I32), t(3, 8, 128)
    assert ta.kv_cache_append(kv, kv, pos=pos, **c) == (c["k_cache"], c["v_cache"])
    assert ta.qk_norm_rope_append(t(3, 8, 128), kv, kv, pos=pos, out=out, cos_sin=t(99, 64, dtype=F32), interleaved=True, **c) == (
        out, c["k_cache"], c["v_cache"])
    assert not calls.made
    (_, append), (_, rope) = calls.calls[-2:]
    assert [n for n, _ in calls.calls[-2:]] == ["qk_norm_rope_append"] * 2
    # without queries, weights and angles; with the angles' rows, their width and the pairs' order
    assert append[0] is None and append[9:13] == (None, 0, 0, 0) and append[18] == 2 and append[24] == 0
    assert rope[10:13] == (99, 64, 1) and rope[18] == 2 and rope[22:27] == (3, 3, 8, 2, 128)


def test_small_workspaces_are_refused(calls):
    """By the library, which gets their size; another type by the binding."""
    args = t(4, 100000), t(4, dtype=F32)
    ta.sample_logits(*args, token=t(4, dtype=I32), logp=t(4, dtype=F32), workspace=t(100, dtype=U8))
    assert calls.calls[-1][1][-2] == 100
    with pytest.raises(TypeError):
        ta.sample_logits(*args, token=t(4, dtype=I32), logp=t(4, dtype=F32), workspace=t(1 << 20, dtype=F32))


def test_product_without_memory_for_the_shares(calls, monkeypatch):
    def full(*args):
        raise torch.OutOfMemoryError("full")

    monkeypatch.setattr(ta, "_scratch", full)
    product(64, 4096, 4096)
    assert calls.calls[-1][1][11] == 0            # a strip each
    with pytest.raises(torch.OutOfMemoryError):
        product(64, 4096, 4096, num_parts=256)
