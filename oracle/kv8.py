"""Oracle of the 8-bit paged K/V cache, float64 (TEST INFRASTRUCTURE ONLY).

A page of 16 positions of one KV head is a block.  A finished block holds e4m3 codes x / s, s the smallest power of two
(2^-100 at least) that brings the block's largest magnitude to 448 or less; a block with a value that is not finite has
s = NaN and codes 0.  Everything behind the last finished page is bf16.
"""
from __future__ import annotations

import numpy as np

from .drafter import rope

PAGE = 16


def e4m3_values() -> np.ndarray:
    """The 127 magnitudes of e4m3 (1 sign, 4 exponent, 3 mantissa bits, bias 7; code 127 is NaN), by code."""
    out = []
    for code in range(127):
        e, m = code >> 3, code & 7
        out.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return np.array(out)


_E4M3 = e4m3_values()


def e4m3_decode(code: np.ndarray) -> np.ndarray:
    """Values of uint8 codes (code 127 and 255: NaN)."""
    code = np.asarray(code)
    mag = np.append(_E4M3, np.nan)[code & 127]
    return np.where(code & 128, -mag, mag)


def e4m3_encode(x: np.ndarray) -> np.ndarray:
    """Nearest code of each finite value, ties to the even code, values past 448 to 448; the sign of zero is kept."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(_E4M3, a), 1, 126)
    up, down = _E4M3[hi] - a, a - _E4M3[hi - 1]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def block_scale(x: np.ndarray) -> float:
    if not np.isfinite(x).all():
        return np.nan
    a = np.abs(x).max()
    k = -100
    while a > 448.0 * 2.0 ** k:
        k += 1
    return 2.0 ** k


def encode_block(x: np.ndarray):
    """Codes [16, hd] and scale of a block [16, hd]."""
    s = block_scale(x)
    if np.isnan(s):
        return np.zeros(x.shape, np.uint8), s
    return e4m3_encode(x / s), s


def place_k(code: np.ndarray) -> np.ndarray:
    """Codes [16, hd] in the order of a K page."""
    hd = code.shape[1]
    out = np.empty(16 * hd, np.uint8)
    for t in range(16):
        for d in range(hd):
            out[((t // 8) * (hd // 16) + d // 16) * 128 + (t % 8) * 16 + d % 16] = code[t, d]
    return out


def place_v(code: np.ndarray) -> np.ndarray:
    return np.ascontiguousarray(code.T).reshape(-1)


def as_cached(rows: np.ndarray, length: int) -> np.ndarray:
    """Rows [length, Hkv, hd] of one sequence and layer as attention reads them: finished pages through 8 bits."""
    out = np.array(rows[:length], np.float64)
    for p in range(length // PAGE):
        for h in range(out.shape[1]):
            sl = np.s_[p * PAGE:(p + 1) * PAGE, h]
            code, s = encode_block(out[sl])
            out[sl] = e4m3_decode(code) * s
    return out


def rotate_rows(x: np.ndarray, first: int, theta: float) -> np.ndarray:
    """Rows [n, heads, hd] turned to positions first, first + 1, ..."""
    return np.stack([rope(np.asarray(r, np.float64), first + i, theta) for i, r in enumerate(x)]) if len(x) else x


def attend(q: np.ndarray, keys: np.ndarray, values: np.ndarray) -> np.ndarray:
    """q [n, Hq, hd] of the newest n positions of keys, values [T, Hkv, hd]; causal."""
    n, Hq, hd = q.shape
    T, Hkv, _ = keys.shape
    out = np.zeros(q.shape)
    for j in range(n):
        m = T - n + j + 1
        for h in range(Hq):
            s = keys[:m, h // (Hq // Hkv)] @ q[j, h] / np.sqrt(hd)
            w = np.exp(s - s.max())
            out[j, h] = (w / w.sum()) @ values[:m, h // (Hq // Hkv)]
    return out
