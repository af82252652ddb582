"""The documented limits of the serving calls, on both sides, on the CPU (fake addresses:
what passes the limits is refused for an overlap)."""
import os

import pytest

from paper_2504_17577_amd import tileattn as ta
from test_serving_abi import APPEND, KC

pytestmark = pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="fake-pointer validation cases run only without a GPU")


@pytest.mark.parametrize("Hkv,D", [(1, 64), (8, 128), (1 << 10, 64)])
def test_most_new_tokens(Hkv, D):
    """T Hkv D up to 2^34 - 1024."""
    row = Hkv * D
    T = ((1 << 34) - 1024) // row
    for n, status in ((T, 6), (T + -(-1024 // row), 2)):
        a = dict(APPEND, T=n, Hkv=Hkv, D=D, k_stride=row, v_stride=row, K=KC)
        assert ta.lib().kv_cache_append(*a.values()) == status, n
