"""The serving calls' host logic on the CPU, with stand-ins for GPU tensors and
streams and the C calls recorded (test_binding.py's): workspaces come from the
launch stream's pool, outputs from the current one's; defaults; no memory."""
import pytest

torch = pytest.importorskip("torch")

from paper_2504_17577_amd import tileattn as ta  # noqa: E402
from test_binding import BF16, F32, FakeLib, FakeStream, FakeTensor, fake  # noqa: E402, F401

I32 = torch.int32


class Strided(FakeTensor):
    def stride(self, i=None):
        s = [1]
        for n in reversed(self.shape[1:]):
            s.insert(0, s[0] * n)
        return tuple(s) if i is None else s[i]


def t(*shape, dtype=BF16):
    x = Strided(shape, dtype)
    x.shape = torch.Size(shape)
    return x


@pytest.fixture
def calls(fake, monkeypatch):  # noqa: F811
    monkeypatch.setattr(FakeLib, "LAUNCHES", FakeLib.LAUNCHES + ("kv_cache_append", "attn_decode_paged", "gemm_bf16_epilogue"))
    return fake


def attn(stream, cap, **kw):
    cache = t(10, 2, 64, 128)
    return ta.attn_decode_paged(t(3, 8, 128), cache, cache, t(3, cap // 64, dtype=I32), t(3, dtype=I32), stream=stream,
                                out=t(3, 8, 128, dtype=F32), lse=t(3, 8, dtype=F32), **kw)


@pytest.mark.parametrize("side", [True, False], ids=["side", "current"])
def test_workspaces_are_allocated_on_the_launch_stream(calls, side):
    s = FakeStream() if side else None
    attn(s, 64000)
    ta.gemm_bf16_epilogue(t(8, 4096), t(4096, 4096), out=t(8, 4096, dtype=F32), stream=s)
    assert [m.dtype for m in calls.made] == [torch.uint8] * 2 and all(m.stream is s for m in calls.made)
    assert [m.numel() for m in calls.made] == [ta.attn_paged_workspace_bytes(8, 2, 128, ta.attn_paged_plan(3, 8, 2, 128, 64, 1000)),
                                               ta.gemm_epilogue_workspace_bytes(8, 4096, 4096, ta.gemm_epilogue_plan(8, 4096, 4096))]
    assert [a[-1] for _, a in calls.calls] == [0x5000 if side else 0] * 2


def test_calls_that_need_no_workspace_allocate_none(calls):
    attn(None, 256)
    ta.gemm_bf16_epilogue(t(8, 64), t(64, 4096), out=t(8, 4096, dtype=F32))
    k = t(3, 2, 128)
    cache = t(10, 2, 64, 128)
    assert ta.kv_cache_append(k, k, cache, cache, t(3, 4, dtype=I32), t(3, dtype=I32)) == (cache, cache)
    assert not calls.made and [n for n, _ in calls.calls] == ["attn_decode_paged", "gemm_bf16_epilogue", "kv_cache_append"]


def test_a_small_workspace_is_refused(calls):
    """By the library, which gets its size; another type by the binding."""
    attn(None, 64000, workspace=t(100, dtype=torch.uint8))
    assert calls.calls[-1][1][-2] == 100
    with pytest.raises(TypeError):
        attn(None, 64000, workspace=t(1 << 24, dtype=F32))


def test_product_without_memory_for_the_ranges(calls, monkeypatch):
    def full(*args):
        raise torch.OutOfMemoryError("full")

    monkeypatch.setattr(ta, "_scratch", full)
    args = t(8, 4096), t(4096, 4096)
    out = t(8, 4096, dtype=F32)
    assert ta.gemm_bf16_epilogue(*args, out=out) is out
    assert calls.calls[-1][1][10] == 1            # one range
    with pytest.raises(torch.OutOfMemoryError):
        ta.gemm_bf16_epilogue(*args, out=out, num_splits=5)
