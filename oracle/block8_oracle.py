"""CPU reference, in numpy and 64 bits, of the norm and of the 8-bit block format.  Independent of the HIP library; used only by tests.

The format: blocks of 128 values along the last axis (or 128 x 128 along the last two) share 2^e, the smallest power of two under which the
block's largest magnitude is at most 448, and at least 2^-126; a value is stored as the e4m3 number nearest to v / 2^e, ties to even.  e4m3: sign, 4
exponent bits with bias 7, 3 mantissa bits; 448 the largest value, 2^-9 the smallest.
"""
from __future__ import annotations

import numpy as np

BLOCK, TOP = 128, 448.0


def e4m3_table() -> np.ndarray:
    """The values of the 256 codes (NaN for 0x7f and 0xff)."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e.astype(np.float64) - 10))
    v[(c & 127) == 127] = np.nan
    return np.where(c >> 7, -v, v)


def round_e4m3(v: np.ndarray) -> np.ndarray:
    """float64 values of magnitude at most 448, to the nearest e4m3 value, ties to the even mantissa: by searching the table."""
    mags = e4m3_table()[:127]
    a = np.abs(v)
    hi = np.clip(np.searchsorted(mags, a), 1, 126)
    lo = hi - 1
    dl, dh = a - mags[lo], mags[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.copysign(mags[code], v)


def exponent_of(amax: float) -> int:
    """e by trying powers of two."""
    e = -126
    while amax > TOP * 2.0 ** e:
        e += 1
    return e


def quantize(v: np.ndarray, blocks: bool):
    """(values as the format holds them, exponents [.., R or ceil(R / 128), ceil(K / 128)]) of float64 v [.., R, K]."""
    R, K = v.shape[-2:]
    step = BLOCK if blocks else 1
    out = np.empty_like(v)
    exps = np.empty((*v.shape[:-2], -(-R // step), -(-K // BLOCK)), dtype=np.int64)
    for lead in np.ndindex(*v.shape[:-2]):
        for i in range(exps.shape[-2]):
            for j in range(exps.shape[-1]):
                at = (*lead, slice(i * step, (i + 1) * step), slice(j * BLOCK, (j + 1) * BLOCK))
                e = exponent_of(np.abs(v[at]).max())
                exps[(*lead, i, j)] = e
                out[at] = round_e4m3(v[at] / 2.0 ** e) * 2.0 ** e
    return out, exps


def rms_norm(x, residual, weight, eps):
    h = x if residual is None else x + residual
    r = 1.0 / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps)
    return h, h * r * (1.0 if weight is None else weight)


def rms_norm_backward(dy, dh, h, weight, eps):
    M = h.shape[1]
    r = 1.0 / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps)
    g = dy if weight is None else dy * weight
    dx = r * g - h * r ** 3 * np.sum(g * h, axis=1, keepdims=True) / M
    return (dx if dh is None else dx + dh), np.sum(dy * h * r, axis=0)
