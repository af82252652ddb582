"""A bf16 O of attn_decode_paged is the fp32 one of the same call, rounded once to nearest:
the softmax weights enter the product with V with all their 24 bits for both.  (The same
additions in the same order, so equal bit for bit; fp32 results are held to the oracle in
test_serving_gpu.py.)"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, E4M3, I32 = torch.bfloat16, torch.float8_e4m3fn, torch.int32


@pytest.fixture(scope="module")
def ta():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2504_17577_amd import tileattn
    tileattn.lib()
    return tileattn


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("B,group,D,P,top", [
    (40, 4, 64, 16, 37), (30, 1, 128, 16, 2), (8, 16, 128, 64, 700), (6, 24, 64, 32, 500), (6, 33, 128, 16, 300), (2, 3, 128, 256, 20000),
])
def test_bf16_result_is_the_fp32_one_rounded(ta, B, group, D, P, top, e4m3):
    g = torch.Generator(device="cuda").manual_seed(top + D)
    per, Hkv = -(-top // P), 2
    kc, vc = (torch.randn(B * per, Hkv, P, D, generator=g, device="cuda").to(E4M3 if e4m3 else BF16) for _ in range(2))
    table = torch.randperm(B * per, generator=g, device="cuda").to(I32).view(B, per)
    lens = torch.randint(0, top + 1, (B,), generator=g, device="cuda").to(I32)
    lens[0] = top
    q = torch.randn(B, Hkv * group, D, generator=g, device="cuda").to(BF16)
    for parts in (None, 0, 1, 37):
        print(f"  parts {parts}", flush=True)
        o32, l32 = ta.attn_decode_paged(q, kc, vc, table, lens, num_parts=parts)
        o16, l16 = ta.attn_decode_paged(q, kc, vc, table, lens, num_parts=parts, out_dtype=BF16)
        assert torch.equal(l16, l32)
        off = o16 != o32.to(BF16)
        assert not off.any(), f"{int(off.sum())} of {off.numel()}"
