"""The workspace of sample_logits goes by the logits' type: a row of bf16 is half as long
in memory, and one workgroup takes it whole where fp32's needs slices.  Sizes and the
binding on the CPU, calls without a workspace on the GPU."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2504_17577_amd import tileattn as ta  # noqa: E402
from test_binding import BF16, F32, fake  # noqa: E402, F401
from test_more_serving_binding import calls  # noqa: E402, F401
from test_serving_binding import t  # noqa: E402

I32 = torch.int32


def test_sizes():
    """None where a row is one slice: 17408 chunks of 16 bytes, two of them for a row's ends."""
    size = ta.sample_workspace_bytes
    for B in (128, 1000, 1 << 16):
        assert size(B, 69627, F32) == 0 < size(B, 69628, F32)
        assert size(B, 139255, BF16) == 0 < size(B, 139256, BF16)
    for B in (1, 127, 128):
        assert size(B, 32768, F32) == size(B, 32768, BF16) == 0
    assert size(127, 32769, BF16) > 0 and size(128, 32769, F32) == 0
    for B in (1, 7, 60, 127, 128, 5000, 1 << 16):
        for V in (1, 1000, 32769, 70000, 131072, 139256, 152064, 300000, 1 << 20):
            assert size(B, V, BF16) <= size(B, V, F32) == size(B, V)
    for dtype in (BF16, F32):
        for bad in [(0, 10), (10, 0), ((1 << 16) + 1, 10), (10, (1 << 20) + 1)]:
            with pytest.raises(ta.TileAttnError):
                size(*bad, dtype)
    assert ta.lib().sample_logits_workspace_bytes(1, 1, 0, ctypes.POINTER(ctypes.c_size_t)()) == 1


def test_the_binding_allocates_by_type(calls):  # noqa: F811
    for dtype, n in ((BF16, 0), (F32, 1)):
        calls.made.clear()
        ta.sample_logits(t(256, 131072, dtype=dtype), t(256, dtype=F32), token=t(256, dtype=I32), logp=t(256, dtype=F32))
        assert len(calls.made) == n
    assert calls.made[0].numel() == ta.sample_workspace_bytes(256, 131072, F32)


@pytest.mark.gpu
@pytest.mark.parametrize("B,V,dtype", [(256, 131072, BF16), (130, 139255, BF16), (128, 69627, F32), (3, 32768, F32)])
def test_calls_that_need_no_workspace_take_none(B, V, dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    g = torch.Generator(device="cuda").manual_seed(V)
    x, u = torch.randn(B, V, generator=g, device="cuda").to(dtype), torch.rand(B, generator=g, device="cuda")
    k = torch.full((B,), 40, dtype=I32, device="cuda")
    for top_k in (None, k):
        want = ta.sample_logits(x, u, top_k=top_k, workspace=torch.empty(1 << 26, dtype=torch.uint8, device="cuda"))
        for none in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
            got = ta.sample_logits(x, u, top_k=top_k, workspace=none)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
