"""Plain numpy float64 oracle of the operators around chunks of new tokens: 8-bit rows, causal attention of a chunk over a cache.

Written from the definitions, one sequence and head at a time; imports nothing from the product.
"""
from __future__ import annotations

import numpy as np

INT8_LARGEST, E4M3_LARGEST = 127.0, 448.0


def e4m3_values() -> np.ndarray:
    """The value of every e4m3 byte: sign, 4 exponent bits (bias 7), 3 mantissa bits; exponent 0: no leading one; all ones: NaN."""
    out = np.zeros(256)
    for code in range(256):
        sign, e, m = (-1.0 if code & 0x80 else 1.0), (code >> 3) & 15, code & 7
        v = m / 8.0 * 2.0 ** -6 if e == 0 else (1.0 + m / 8.0) * 2.0 ** (e - 7)
        out[code] = np.nan if e == 15 and m == 7 else sign * v
    return out


def _nearest(y: np.ndarray, grid: np.ndarray) -> np.ndarray:
    """Index of the entry of the ascending grid of non-negative values that is nearest to each y >= 0, ties to the even index."""
    hi = np.clip(np.searchsorted(grid, y, side="left"), 1, len(grid) - 1)
    lo = hi - 1
    dl, dh = y - grid[lo], grid[hi] - y
    return np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))


def quantise(x: np.ndarray, fmt: str):
    """Rows x [..., d] -> (codes as stored bytes uint8, scales float32)."""
    x = np.asarray(x, np.float64)
    largest = INT8_LARGEST if fmt == "int8" else E4M3_LARGEST
    top = np.abs(x).max(axis=-1)
    with np.errstate(invalid="ignore", over="ignore"):
        scale = (top / largest).astype(np.float32)
    bad = ~np.isfinite(top)
    scale[bad] = np.nan
    s = np.where(bad | (scale == 0), 1.0, scale.astype(np.float64))[..., None]
    y = np.where(bad[..., None] | (scale == 0)[..., None], 0.0, x) / s
    # (a code's magnitude counts up with its value in both formats: an even index is an even last bit)
    grid = np.arange(128.0) if fmt == "int8" else e4m3_values()[:0x7f]
    mag = _nearest(np.minimum(np.abs(y), largest), grid)
    if fmt == "int8":
        codes = (np.sign(y) * mag).astype(np.int8).view(np.uint8)
    else:
        codes = (mag + np.where(np.signbit(y), 0x80, 0)).astype(np.uint8)
    return codes, scale


def values(codes: np.ndarray, fmt: str) -> np.ndarray:
    return codes.view(np.int8).astype(np.float64) if fmt == "int8" else e4m3_values()[codes]


def dequantise(codes: np.ndarray, scale: np.ndarray, fmt: str) -> np.ndarray:
    return values(codes, fmt) * scale.astype(np.float64)[..., None]


def chunk_attend(q: np.ndarray, K: np.ndarray, V: np.ndarray):
    """q [n][G][d], the last n of N tokens; K, V [N][d], all float64.  Returns O [n][G][d], and what bounds its error: the weighted
    mean of |V| [n][G][d] and the largest sum of |q_i K_i| / sqrt(d) over the tokens seen [n][G]."""
    n, G, d = q.shape
    N = K.shape[0]
    O, A, L = np.zeros((n, G, d)), np.zeros((n, G, d)), np.zeros((n, G))
    for i in range(n):
        seen = N - n + i + 1
        for g in range(G):
            x = K[:seen] @ q[i, g] / np.sqrt(d)
            w = np.exp(x - x.max())
            w /= w.sum()
            O[i, g] = w @ V[:seen]
            A[i, g] = w @ np.abs(V[:seen])
            L[i, g] = (np.abs(K[:seen]) @ np.abs(q[i, g])).max() / np.sqrt(d)
    return O, A, L
