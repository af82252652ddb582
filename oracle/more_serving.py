"""Float64 reference of the serving step's other calls: 4-bit numbers, norm and
rotation of queries and keys, and the choice of the next token.

TEST INFRASTRUCTURE, like the rest of this package: plain definitions over numpy
arrays, sharing no code with the kernels.
"""
from __future__ import annotations

import numpy as np

GROUP = 32
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def mx_values(codes, scales) -> np.ndarray:
    """The float64 numbers of codes [.., n / 2] with scale bytes [.., n / 32]."""
    nib = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    x = np.where(nib >= 8, -1.0, 1.0) * E2M1[nib & 7]
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127.0))
    return x * np.repeat(s, GROUP, -1)


def mx_pack(x) -> tuple[np.ndarray, np.ndarray]:
    """(codes, scale bytes) of float32 x [.., n]: for every 32 the power of two that puts
    the largest between 3.5 and 7, the nearest e2m1 (ties to the even code), 6 at most."""
    g = np.asarray(x, np.float32).astype(np.float64).reshape(*np.shape(x)[:-1], -1, GROUP)
    nan = np.isnan(g).any(-1)
    g = np.clip(np.where(nan[..., None], 0.0, g), -np.finfo(np.float32).max, np.finfo(np.float32).max)
    top = np.abs(g).max(-1)
    m, e = np.frexp(np.where(top == 0, 1.0, top))          # top = m 2^e, 0.5 <= m < 1
    e = np.where(top == 0, -1000, e - 1 - 2 + (m >= 0.875))
    e = np.clip(e, -126, 125)
    y = g / np.exp2(e)[..., None]
    a = np.minimum(np.abs(y), 6.0)
    hi = np.minimum(np.searchsorted(E2M1, a), 7)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - E2M1[lo], E2M1[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi) | (np.signbit(y) << 3)
    code = np.where(nan[..., None], 0, code).reshape(*np.shape(x)[:-1], -1).astype(np.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), np.where(nan, 255, e + 127).astype(np.uint8)


def norm_rope(x, pos, weight=None, eps=1e-6, cos_sin=None, interleaved=False):
    """(y, the sizes that its rounding errors scale with) of x [T, H, D], normed and
    rotated; pos [T] within cos_sin's rows."""
    x = np.asarray(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    y, size = x.copy(), np.abs(x)
    if cos_sin is not None:
        rot = cos_sin.shape[1]
        n = rot // 2
        c, s = cos_sin[pos][:, None, :n].astype(np.float64), cos_sin[pos][:, None, n:].astype(np.float64)
        ia, ib = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, n), slice(n, rot))
        a, b = x[..., ia], x[..., ib]
        y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
        size[..., ia], size[..., ib] = np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)
    return y, size


def sample(x, u, temperature=1.0, top_k=0, top_p=np.inf, min_p=0.0, error=0.0):
    """(tokens, logp of each) for one row of logits: the answer, or all of them that there
    are if sums of weights are off by up to `error`."""
    x = np.asarray(x, np.float64)
    V = len(x)
    best = x.max() if not np.isnan(x).any() else np.nan
    if not np.isfinite(best):
        return [-1], [np.nan]
    greedy = not temperature > 0
    T = 1.0 if greedy else min(max(float(temperature), 1e-30), 1e30)
    w = np.exp((x - best) / T)
    order = np.lexsort((np.arange(V), -(x + 0.0)))
    ws = w[order]
    k = 1 if greedy else min(V, top_k) if top_k > 0 else V
    before = np.concatenate([[0.0], np.cumsum(ws)[:-1]])[:k]
    total = ws[:k].sum()
    u = min(max(float(u), 0.0), 1.0 - 2.0 ** -53)
    tokens = set()

    def kept(off):
        keep = np.ones(k, bool)
        if top_p < 1 or np.isnan(top_p):
            keep &= before < top_p * total + off
        if not min_p <= 0:
            keep &= ws[:k] >= min_p - off
        return max(1, int(keep.sum()))

    low, high = (kept(-error), kept(error)) if error else (kept(0.0),) * 2
    for n in range(low, high + 1):
        some = np.sort(order[:n])
        upto = np.cumsum(w[some])
        last = int(np.searchsorted(upto, upto[-1]))      # (the last that counts)
        at = [min(last, int(np.searchsorted(upto, u * upto[-1] + d, side="right"))) for d in (-error, error)]
        tokens.update(int(t) for t in some[at[0]:at[1] + 1] if w[t] > 0)
    tokens = sorted(tokens)
    return tokens, [(x[t] - best) / T - np.log(w.sum()) for t in tokens]
