"""Pins of the oracle's 4-bit numbers and of its norm and rotation: closed forms."""
import numpy as np

from oracle import more_serving as ms


def test_values():
    codes = np.array([[0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE] * 2], np.uint8)
    x = ms.mx_values(codes, np.array([[127]], np.uint8))[0]
    half = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    assert x.tolist() == (half + [-v for v in half]) * 2 and np.signbit(x[8])
    assert (ms.mx_values(codes, np.array([[130]], np.uint8))[0] == 8 * x).all()
    assert np.isnan(ms.mx_values(codes, np.array([[255]], np.uint8))).all()


def test_pack_finds_the_nearest():
    """Against every one of the 16 numbers, at the scale that the rule names."""
    x = np.random.default_rng(0).standard_normal((500, 64)).astype(np.float32) * np.exp2(np.arange(500) % 40 - 20)[:, None].astype(np.float32)
    codes, scales = ms.mx_pack(x)
    v = ms.mx_values(codes, scales)
    top = np.abs(x.reshape(500, 2, 32)).max(-1) / np.exp2(scales - 127.0)
    assert (top >= 3.5).all() and (top < 7).all()
    s = np.repeat(np.exp2(scales - 127.0), 32, -1)
    every = np.concatenate([ms.E2M1, -ms.E2M1])
    best = np.abs(x[..., None] - every * s[..., None]).min(-1)
    assert (np.abs(v - x) == best).all()


def test_pack_of_ties_and_specials():
    x = np.zeros((7, 32), np.float32)
    x[0, :8] = [4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -5 / 2]
    x[1, :2] = [6.999, 5]
    x[2, :2] = [7, 5]
    x[3, :2] = [np.inf, -np.inf]
    x[4, 3] = np.nan
    x[5, 0] = 1e-45
    codes, scales = ms.mx_pack(x)
    v = ms.mx_values(codes, scales)
    assert v[0, :8].tolist() == [4, 0, 1, 1, 2, 2, 4, -2] and scales[0] == 127
    assert v[1, :2].tolist() == [6, 4] and scales[1] == 127 and v[2, :2].tolist() == [8, 4] and scales[2] == 128
    assert v[3, :2].tolist() == [6 * 2.0 ** 125, -6 * 2.0 ** 125] and scales[3] == 252
    assert scales[4] == 255 and (codes[4] == 0).all() and scales[5] == 1 and (v[5] == 0).all() and scales[6] == 1
    assert (ms.mx_values(*ms.mx_pack(v[:3])) == v[:3]).all()


def test_norm_and_rotation():
    x = np.random.default_rng(1).standard_normal((3, 2, 64))
    n, _ = ms.norm_rope(x, np.zeros(3, int), np.ones(64), 0.0)
    assert np.allclose((n * n).mean(-1), 1)
    a = np.array([0.3, 1.1, 2.0])[:, None] * np.ones(16)
    cs = np.concatenate([np.cos(a), np.sin(a)], 1)
    pos = np.array([2, 0, 1])
    for inter in (False, True):
        y, _ = ms.norm_rope(x, pos, cos_sin=cs, interleaved=inter)
        assert np.allclose((y * y).sum(-1), (x * x).sum(-1)) and (y[..., 32:] == x[..., 32:]).all()
        z = x[..., 0:32:2] + 1j * x[..., 1:32:2] if inter else x[..., :16] + 1j * x[..., 16:32]
        z = z * np.exp(1j * a[pos])[:, None]
        w = y[..., 0:32:2] + 1j * y[..., 1:32:2] if inter else y[..., :16] + 1j * y[..., 16:32]
        assert np.allclose(z, w)


def test_sample():
    x = np.log([4.0, 1.0, 2.0, 1.0])
    one = lambda *a, **k: ms.sample(*a, **k)[0]    # noqa: E731
    for u, t in ((0.0, 0), (0.49, 0), (0.51, 1), (0.63, 2), (0.9, 3)):
        assert one(x, u) == [t] == one(x, u, error=1e-3)
    assert np.isclose(ms.sample(x, 0.7)[1][0], np.log(0.25))
    assert one(x, 0.9, top_k=3) == [2] and one(x, 0.6, top_k=3) == [1]      # order 0, 2, 1, 3
    assert one(x, 0.99, top_p=0.5) == [0] and one(x, 0.99, top_p=0.51) == [2]
    assert one(x, 0.99, top_p=0.499, error=0.01) == [0, 2] and one(x, 0.501, error=0.01) == [0, 1]
    assert one(x, 0.99, min_p=0.3) == [2] and one(x, 0.99, min_p=0.6) == [0]
    assert one(x, 0.99, top_p=0.0) == [0] and one(x, 0.99, min_p=2.0) == [0] and one(x, 0.99, min_p=np.nan) == [0]
    assert one([1.0, 3.0, 3.0], 0.9, 0.0) == [1] and one(x, 0.9, top_p=np.nan) == [0]
    assert one(x, 0.7, temperature=0.5) == [0] and one(x, 0.8, temperature=0.5) == [2]   # 16, 1, 4, 1
    assert one([-np.inf, 0.0, -np.inf], 0.99) == [1]
    for bad in ([np.nan, 1.0], [np.inf, 0.0], [-np.inf, -np.inf]):
        assert one(bad, 0.5) == [-1]
