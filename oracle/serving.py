"""Float64 reference of a decoder's serving step: new tokens into a paged
key/value cache, attention of one new token per sequence over it, and the matrix
product with bias, activation and residual.

TEST INFRASTRUCTURE, like the rest of this package: plain definitions over numpy
arrays, sharing no code with the kernels.
"""
from __future__ import annotations

import math

import numpy as np

E4M3_MAX = 448.0


def e4m3_values() -> np.ndarray:
    """The values of the 256 e4m3 codes (OCP: no infinities, NaN at 0x7f and 0xff)."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((e == 15) & (m == 7), np.nan, v)
    return np.where(c >> 7, -v, v)


def e4m3_codes(x) -> np.ndarray:
    """The codes nearest to x (ties to the even code), clamped to +-448; NaN to 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    pos = e4m3_values()[:127]                 # 0 .. 448, increasing
    a = np.minimum(np.abs(x), E4M3_MAX)
    nan = np.isnan(a)
    a = np.where(nan, 0.0, a)
    hi = np.minimum(np.searchsorted(pos, a), 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - pos[lo], pos[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = np.where(nan, 0x7F, code | (np.signbit(x) << 7))
    return code.astype(np.uint8)


def place(table, num_pages, page_size, seq, pos):
    """(page, row in it) of a position, or None where there is none."""
    B, per = table.shape
    if not (0 <= seq < B and 0 <= pos < per * page_size):
        return None
    page = int(table[seq, pos // page_size])
    return (page, pos % page_size) if 0 <= page < num_pages else None


def append(new, cache, table, pos, seq=None, scale=None):
    """A copy of cache [num_pages, Hkv, P, D] (bfloat16 bits, or e4m3 codes) with the
    tokens new [T, Hkv, D] (bfloat16 bits) written; e4m3 from x / scale in float32."""
    out = cache.copy()
    num_pages, Hkv, P, _ = cache.shape
    for t in range(len(new)):
        at = place(table, num_pages, P, t if seq is None else int(seq[t]), int(pos[t]))
        if at is None:
            continue
        row = new[t]
        if cache.dtype == np.uint8:
            x = (row.astype(np.uint32) << 16).view(np.float32)
            s = np.ones(Hkv, np.float32) if scale is None else scale.astype(np.float32)
            with np.errstate(all="ignore"):
                row = e4m3_codes(x / s[:, None])
        out[at[0], :, at[1]] = row
    return out


def attn_paged(q, k, v, table, lens, scale, k_scale=None, v_scale=None):
    """(O, LSE, tolerance of an exact-product fp32 evaluation) for float64 q [B, Hq, D]
    and caches k, v [num_pages, Hkv, P, D].  The tolerance bounds, row by row, the
    error of fp32 dot products of D terms summed in any order (2^-24 each), of the
    exponentials (2^-21) and of fp32 sums over the keys, for |V| at its largest."""
    B, Hq, D = q.shape
    num_pages, Hkv, P, _ = k.shape
    g = Hq // Hkv
    o, lse = np.zeros((B, Hq, D)), np.full((B, Hq), -np.inf)
    tol, tol_lse = np.zeros((B, Hq)), np.zeros((B, Hq))
    for b in range(B):
        n = int(lens[b])
        if n == 0:
            continue
        where = [place(table, num_pages, P, b, t) for t in range(n)] if n > 0 else [None]
        if None in where:
            o[b], lse[b] = np.nan, np.nan
            continue
        pg, row = np.array(where).T
        for h in range(Hkv):
            kk = k[pg, h, row] * (1.0 if k_scale is None else k_scale[h])
            vv = v[pg, h, row] * (1.0 if v_scale is None else v_scale[h])
            for i in range(h * g, (h + 1) * g):
                s = scale * (kk @ q[b, i])
                m = s.max()
                p = np.exp(s - m)
                o[b, i] = (p @ vv) / p.sum()
                lse[b, i] = m + math.log(p.sum())
                d = scale * (D + 4) * 2.0 ** -24 * (np.abs(kk) @ np.abs(q[b, i])).max() \
                    + 2.0 ** -23 * (np.abs(s).max() + abs(m)) + 2.0 ** -21
                tol_lse[b, i] = d + (n + 8) * 2.0 ** -24 + 2.0 ** -22 * abs(lse[b, i])
                tol[b, i] = (2 * d + 2 * (n + 8) * 2.0 ** -24) * np.abs(vv).max()
    return o, lse, tol, tol_lse


def activated(x, name):
    erf = np.vectorize(math.erf)
    if name == "relu":
        return np.maximum(x, 0.0)
    if name == "gelu":
        return 0.5 * x * (1.0 + erf(x / math.sqrt(2.0)))
    if name == "gelu_tanh":
        return 0.5 * x * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3)))
    if name == "silu":
        return x / (1.0 + np.exp(-x))
    return x


def gemm_epilogue(a, b, bias=None, activation="none", residual=None):
    """(C, tolerance of an fp32 evaluation): K exact products summed in any order
    (2^-24 each of the sum of their sizes) and the bias through an activation of
    slope at most 1.13, the activation itself to 2^-20, the residual's sum to 2^-24."""
    x = a @ b
    size = np.abs(a) @ np.abs(b)
    if bias is not None:
        x, size = x + bias, size + np.abs(bias)
    y = activated(x, activation)
    c = y if residual is None else y + residual
    tol = 1.13 * (a.shape[1] + 2) * 2.0 ** -24 * size + 2.0 ** -20 * np.abs(y) + 2.0 ** -24 * np.abs(c) + 1e-30
    return c, tol
