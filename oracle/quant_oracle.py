"""CPU oracle of the caches held in 8 bits -- TEST INFRASTRUCTURE ONLY (numpy, float64, one (batch, kv head) at a time).

e4m3 (sign, 4 exponent bits with bias 7, 3 fraction bits; no infinity, the all-ones pattern is NaN), one power-of-two scale for each
block of 32 slots: value = code * scale.  See the functions for the rules; they are this project's own definition (include/keepkv.h).
"""
from __future__ import annotations

import numpy as np

BLOCK, TOP, LOW, HIGH = 32, 448.0, -110, 120


def _values():
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[c] = np.nan if c & 127 == 127 else (-x if c & 128 else x)
    return v


VALUES = _values()                    # of every code


def scale_of(a: float) -> float:
    """The smallest power of two 2^e, LOW <= e <= HIGH, with a <= TOP * 2^e."""
    for e in range(LOW, HIGH):
        if a <= TOP * 2.0 ** e:
            return 2.0 ** e
    return 2.0 ** HIGH


def encode(x) -> np.ndarray:
    """Nearest code, of two equally near ones the even one; not finite: NaN.  |x| <= TOP where finite."""
    x = np.asarray(x, np.float64)
    pos = VALUES[:127]
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    hi = np.clip(np.searchsorted(pos, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - pos[lo], pos[hi] - a
    c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    c = np.where(a == pos[hi], hi, c) | np.where(np.signbit(x), 128, 0)
    return np.where(np.isfinite(x), c, 127).astype(np.uint8)


def _amax(x) -> float:
    a = np.abs(np.asarray(x, np.float64))
    a = a[np.isfinite(a)]
    return float(a.max()) if a.size else 0.0


def quantize(rows):
    """rows [n, D] -> codes [n, D] uint8, scales [ceil(n / BLOCK)]."""
    rows = np.asarray(rows, np.float64)
    codes = np.zeros(rows.shape, np.uint8)
    scales = []
    for b in range(0, len(rows), BLOCK):
        s = scale_of(_amax(rows[b:b + BLOCK]))
        codes[b:b + BLOCK] = encode(rows[b:b + BLOCK] / s)
        scales.append(s)
    return codes, np.array(scales)


def values(codes, scales):
    """What the codes [n, D] stand for."""
    n = len(codes)
    return VALUES[codes] * np.repeat(np.asarray(scales, np.float64), BLOCK)[:n, None]


def append(codes, scales, new):
    """codes [n, D], scales [ceil(n / BLOCK)], new rows [m, D] -> the grown codes and scales."""
    n, new = len(codes), np.asarray(new, np.float64)
    codes = np.concatenate([codes, np.zeros(new.shape, np.uint8)])
    scales = list(np.asarray(scales, np.float64))
    for b in range(n // BLOCK, (n + len(new) + BLOCK - 1) // BLOCK):
        lo, hi = max(n, b * BLOCK), min(n + len(new), (b + 1) * BLOCK)
        if hi <= lo:
            continue
        s = scale_of(_amax(new[lo - n:hi - n]))
        if lo > b * BLOCK:
            old = scales[b]
            s = max(s, old)
            if s != old:
                codes[b * BLOCK:lo] = encode(VALUES[codes[b * BLOCK:lo]] * (old / s))
            scales[b] = s
        else:
            scales.append(s)
        codes[lo:hi] = encode(new[lo - n:hi - n] / s)
    return codes, np.array(scales)
