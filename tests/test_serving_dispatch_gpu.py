"""Kernels of the serving calls that a call's sizes choose and no other test runs: paged
attention over an 8-bit cache of 128 dims with more than 16 query heads to a K/V head, and
products of few rows by their blocks of 16, with weights on both sides of the 256 MB from
which they are loaded with the non-temporal policy."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_serving_gpu import BF16, F32, Cache, check, reference, ta  # noqa: E402, F401
from test_serving_tiles import check_product  # noqa: E402


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,P", [(17, 1, 16), (64, 2, 64), (40, 1, 128), (33, 1, 32), (192, 2, 16)])
def test_eight_bit_cache_with_many_heads(ta, Hq, Hkv, P, dtype):  # noqa: F811
    lens = [1, 0, 16, 33, 700, 15]
    c = Cache(lens, Hkv, 128, P, True, seed=Hq)
    q = torch.randn(len(lens), Hq + 2, 128, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()[:, 2:]
    ref = reference(q, c, 128 ** -0.5)
    for parts in (None, 0, 1, 5, 512):
        print(f"  parts {parts}", flush=True)
        check(c, *ta.attn_decode_paged(q, *c.args(), **c.scales(), num_parts=parts, out_dtype=dtype), ref)


@pytest.mark.parametrize("dt", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("M", [5, 16, 17, 33, 48, 64])
@pytest.mark.parametrize("N,K", [(1000, 1032), (40000, 4104)])
def test_few_rows_by_their_blocks(M, N, K, dt):
    assert (2 * N * K > 256 << 20) == (N == 40000)
    for splits in (None, 1, 3):
        check_product(M, N, K, splits, dt)
