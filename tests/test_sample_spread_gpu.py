"""sample_logits over rows whose logits lie very close together or very far apart: by
less than the smallest normal number, by a few powers of two more, and up to the whole
range of fp32."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_sample_gpu import BF16, F32, I32, INF, col, compare, ta  # noqa: E402, F401

pytestmark = pytest.mark.gpu

# the least of fp32's and of bf16's denormal numbers, the least normal ones, and those at
# which a quotient of 1023 and the spread leaves fp32 (3e-36)
SPREADS = [2.0 ** -149, 2.0 ** -133, 2.0 ** -126, 1e-37, 2.9e-36, 3.1e-36, 1e-35, 1e-30, 1e30, 3e38]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("B,V", [(3, 2), (3, 150), (3, 1024), (3, 1025), (3, 9000), (3, 40000), (130, 3000), (2, 100001)])
def test_one_logit_apart(ta, B, V, dtype):  # noqa: F811
    """A row of zeros but for one place: the largest, whatever it is larger by, and the first
    of a top-k; the smallest, where it is less by that."""
    for spread in SPREADS:
        at = V * 2 // 3
        x = torch.zeros(B, V, dtype=dtype, device="cuda")
        x[:, at] = spread
        if not float(x[0, at]):
            continue                          # (fp32's denormals in bf16)
        u = np.linspace(0.0, 1 - 2.0 ** -24, B)
        token, _ = ta.sample_logits(x, col(u), col([0.0] * B))
        assert (token == at).all(), (spread, token.tolist())
        token, _ = ta.sample_logits(x, col(u), None, col([1] * B, I32))
        assert (token == at).all(), (spread, token.tolist())
        token, _ = ta.sample_logits(x, col([1 - 2.0 ** -24] * B), None, col([3] * B, I32))
        assert (token == (at if at > 1 or spread > 1 else min(2, V - 1))).all(), (spread, token.tolist())
        rows = slice(0, 3)                    # (the oracle's part)
        for k in (None, 3, min(V, 700)):
            compare(ta, x[rows], u[rows], None, None if k is None else [k] * min(B, 3), unclear=3)
        token, _ = ta.sample_logits(-x, col(u), col([0.0] * B))
        assert (token == 0).all(), (spread, token.tolist())
        token, _ = ta.sample_logits(-x, col([1 - 2.0 ** -24] * B), None, col([V - 1] * B, I32))
        assert (token == (V - 1 if at < V - 1 else V - 2)).all(), (spread, token.tolist())


@pytest.mark.parametrize("V", [77, 1024, 5000, 70001])
def test_logits_within_a_small_spread(ta, V):  # noqa: F811
    """Many different logits, all within it, at temperatures that make them matter and that
    do not; and the whole range of fp32."""
    g = torch.Generator().manual_seed(V)
    for spread in SPREADS[2:]:
        x = (torch.rand(4, V, generator=g) * spread).cuda()
        x[1] -= spread / 2
        x[2, ::2] = -INF
        u = torch.rand(4, generator=g).numpy()
        for T in (None, 1e-30, 1e30, 0.0):
            compare(ta, x, u, None if T is None else [T] * 4, unclear=4)
            compare(ta, x, u, None if T is None else [T] * 4, [20] * 4, [0.9] * 4, unclear=4)
