"""Rotary positions in float64, pair by pair from the definition: pair i turns
by position * freq[i] radians, its dims being (i, i + rot/2) or, interleaved,
(2i, 2i + 1); dims from rot on are copied.  Also the cache row of each new token
of a ragged batch."""

from __future__ import annotations

import math

import numpy as np


def frequencies(rot: int, theta: float, scaling: str = "none", factor: float = 1.0,
                original_context: int = 0, beta_fast: float = 32.0, beta_slow: float = 1.0):
    """(freq [rot/2], factor on the rotated values)."""
    base = theta * factor ** (rot / (rot - 2)) if scaling == "ntk" else theta
    freq, extra = [], 1.0
    for i in range(rot // 2):
        f = 1.0 / base ** (2 * i / rot)
        if scaling == "linear":
            f /= factor
        if scaling == "yarn":
            # Pair j turns beta times in the original context where
            # original_context * theta^(-2j/rot) = 2 pi beta.
            def pair(beta):
                return rot / 2 * math.log(original_context / (2 * math.pi * beta)) / math.log(theta)
            low = max(math.floor(pair(beta_fast)), 0)
            high = min(math.ceil(pair(beta_slow)), rot - 1)
            part = min(max((i - low) / (high - low if high > low else 0.001), 0.0), 1.0)
            f = f * (1 - part) + f / factor * part
            extra = 0.1 * math.log(factor) + 1.0
        freq.append(f)
    return np.array(freq), extra


def rotate(x: np.ndarray, positions, freq, *, interleaved=False, factor=1.0) -> np.ndarray:
    """x [tokens, heads, d] float64."""
    y = x.astype(np.float64).copy()
    half = len(freq)
    for i in range(half):
        i1, i2 = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = np.asarray(positions, np.float64)[:, None] * freq[i]
        c, s = np.cos(angle) * factor, np.sin(angle) * factor
        y[..., i1] = x[..., i1] * c - x[..., i2] * s
        y[..., i2] = x[..., i2] * c + x[..., i1] * s
    return y


def cache_rows(q_starts, kv_lens, tokens: int):
    """(sequence, cache index) of each token; (-1, 0) outside every sequence."""
    rows = [(-1, 0)] * tokens
    for b, n in enumerate(kv_lens):
        first, last = int(q_starts[b]), int(q_starts[b + 1])
        for t in range(first, last):
            rows[t] = (b, int(n) - (last - t))
    return rows
