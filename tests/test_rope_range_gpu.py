"""The norm of qk_norm_rope_append over the whole range of bf16: heads whose squares, or
the sums of them, leave the range of fp32 on either side, with and without eps, beside
ordinary heads, for queries and for keys in every type of cache.  Tolerances as
test_rope_append_gpu.py derives them, and half a step of bf16's denormal numbers
(2^-134)."""
import numpy as np
import pytest

from oracle import more_serving as ms

torch = pytest.importorskip("torch")
from test_rope_append_gpu import BF16, I32, Pool, angles, bits, f64, ta  # noqa: E402, F401

pytestmark = pytest.mark.gpu

# (zeros: of no eps 0 / 0, whose sign as an 8-bit code is nobody's matter)
SIZES = [1.0, 1e15, 2.0 ** 63, 1e20, 1e25, 1e30, 2e37, 1e-10, 2.0 ** -57, 1e-18, 2.0 ** -63, 1e-20, 1e-25, 1e-30, 2.0 ** -125,
         2.0 ** -131, 0.0]


@pytest.mark.parametrize("eps", [0.0, 1e-6, 1e-20, 1e-45, 1e30])
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "mxfp4"])
@pytest.mark.parametrize("D,inter", [(64, False), (128, True)])
def test_norm_over_the_range_of_bf16(ta, D, inter, kind, eps):  # noqa: F811
    T, Hq, Hkv = len(SIZES), 3, 2
    g = torch.Generator().manual_seed(D)
    x = torch.randn(T, Hq + 2 * Hkv, D, generator=g, dtype=torch.float64)
    size = torch.tensor(SIZES if eps else SIZES[:-1] + [1.0], dtype=torch.float64)[:, None, None]
    x = (x.clamp(-4, 4) * size)
    x[:, 1] /= 16                  # (heads of a token differ)
    x[:, 2, 1:] *= 2.0 ** -70      # one number that counts alone
    x[:, Hq, D // 2:] *= 2.0 ** -40
    x = x.to(BF16).cuda()
    assert torch.isfinite(x).all()
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    w = [(torch.randn(D, generator=g) * 0.2 + 1).to(BF16).cuda() for _ in range(2)]
    pool = Pool(T, 1, Hkv, D, 16, kind, seed=1)
    pos = torch.arange(T, dtype=I32) % 16
    cs, pn, eps = angles(16, D), pos.numpy(), float(np.float32(eps))
    y = [ms.norm_rope(f64(t), pn, f64(n), eps, cs.cpu().numpy(), inter) for t, n in ((q, w[0]), (k, w[1]))]
    with np.errstate(over="ignore"):        # (values past the range of fp32 by their scale)
        want = [pool.want(t, s, i, pn, None, [True] * T) for i, (t, s) in enumerate(((y[1][0], pool.ks), (f64(v), pool.vs)))]
    out, _, _ = ta.qk_norm_rope_append(q, k, v, pool.k, pool.v, pool.table, pos.cuda(), cos_sin=cs, q_weight=w[0], k_weight=w[1],
                                       eps=eps, interleaved=inter, k_scale=pool.ks, v_scale=pool.vs)

    def close(got, x, size):
        tol = 20 * 2.0 ** -24 * size + 2.0 ** -8 * np.abs(x) + 2.0 ** -134
        ok = np.abs(got - x) <= tol
        assert ok.all(), [(SIZES[t], int(h)) for t, h in {(int(i[0]), int(i[1])) for i in np.argwhere(~ok)}]

    close(f64(out), *y[0])
    if kind == "bf16":
        page = pool.table[:, 0].long().cpu().numpy()
        close(f64(pool.k)[page, :, pn], *y[1])
    else:
        for a, b in zip(want[0], (pool.k, pool.ks)):
            np.testing.assert_array_equal(bits(b), a)
    for a, b in zip(want[1], (pool.v, pool.vs)):
        np.testing.assert_array_equal(bits(b), a)
