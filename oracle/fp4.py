"""The cache's 4-bit form in float64: 32 dims share a power of two 2^e, and each is one
of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times it, with a sign; two dims a byte, the even one in the
low half; a scale byte is e + 127, or 255 where all 32 are NaN."""

from __future__ import annotations

import math

import numpy as np

SIZES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def decode(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """[..., d / 2] and [..., d / 32] to [..., d]."""
    both = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1]).astype(np.int64)
    x = np.where(both & 8, -SIZES[both & 7], SIZES[both & 7])
    e = np.repeat(scales.astype(np.int64), 32, -1)
    return np.where(e == 255, np.nan, np.ldexp(x, e - 127))


def exponent(largest: float) -> int:
    """The least e in [-125, 125] with largest < 7 * 2^e."""
    if largest == 0.0:
        return -125
    e = max(-125, math.frexp(largest)[1] - 4)
    while e < 125 and not largest < 7.0 * 2.0 ** e:
        e += 1
    return e


def encode(x: np.ndarray):
    """[..., d] to codes and scales: the nearest size, of two as near the even one."""
    groups = np.asarray(x, np.float64).reshape(-1, 32)
    codes = np.zeros(groups.shape, np.int64)
    scales = np.zeros(len(groups), np.int64)
    for i, g in enumerate(groups):
        if not np.isfinite(g).all():
            scales[i] = 255
            continue
        e = exponent(float(np.abs(g).max()))
        scales[i] = e + 127
        away = np.abs(np.abs(g)[:, None] - np.ldexp(SIZES, e)[None])
        near = away == away.min(1, keepdims=True)
        even = near & (np.arange(8) % 2 == 0)
        best = np.where(near.sum(1) > 1, even.argmax(1), near.argmax(1))
        codes[i] = best + 8 * np.signbit(g)
    pair = codes.reshape(*np.shape(x)[:-1], -1, 2)
    return ((pair[..., 0] + 16 * pair[..., 1]).astype(np.uint8),
            scales.reshape(*np.shape(x)[:-1], -1).astype(np.uint8))
