"""The parts that the attention over 4 bits is planned in: no more than run at once."""
import pytest

from paper_2504_17577_amd import tileattn as ta


@pytest.mark.parametrize("D", [64, 128])
def test_parts_by_the_heads_of_a_workgroup(D):
    for group in range(1, 200):
        rows = -(-group // -(-group // 32))        # the query heads of a workgroup
        for B, Hkv, page, per in ((1, 1, 64, 2000), (64, 2, 16, 1024), (4, 8, 64, 128)):
            assert ta.attn_paged_mxfp4_plan(B, group * Hkv, Hkv, D, page, per) == (768 if rows <= 16 else 512)
        assert ta.attn_paged_mxfp4_plan(5, group * 2, 2, D, 64, 4) == 0 == ta.attn_paged_plan(5, group * 2, 2, D, 64, 4)
