"""Attention of the new tokens of a ragged batch over a cache, in float64, one row
at a time over the keys that row sees: token i of n new ones sits at position
p = kv - n + i and sees the keys up to the end of its block of `mask_block`
positions (all for 0), none if p < 0."""

from __future__ import annotations

import math

import numpy as np


def seen(kv: int, n: int, i: int, mask_block: int) -> int:
    p = kv - n + i
    if p < 0:
        return 0
    return kv if mask_block == 0 else min(kv, (p // mask_block + 1) * mask_block)


def gather(cache: np.ndarray, table, b: int, n: int, page: int) -> np.ndarray:
    """The first n cached tokens of sequence b, [n, Hkv, d]."""
    if not page:
        return cache[b, :n]
    return np.stack([cache[int(table[b, t // page]), t % page] for t in range(n)]) if n else cache[0, :0]


def chunk_attention(q, k_cache, v_cache, table, q_starts, kv_lens, *, mask_block=1, page=0, scale=0.0):
    """(out [tokens, Hq, d], lse [Hq, tokens], weighted |v| [tokens, Hq, d], largest
    sum of |q k| scale [Hq, tokens]); rows outside q_starts' range are NaN."""
    T, hq, d = q.shape
    hkv = k_cache.shape[2]
    scale = scale or 1.0 / math.sqrt(d)
    out = np.full((T, hq, d), np.nan)
    lse = np.full((hq, T), np.nan)
    size = np.full((T, hq, d), np.nan)
    spread = np.zeros((hq, T))
    for b, kv in enumerate(kv_lens):
        first, last = int(q_starts[b]), int(q_starts[b + 1])
        k = gather(k_cache, table, b, int(kv), page).astype(np.float64)
        v = gather(v_cache, table, b, int(kv), page).astype(np.float64)
        for t in range(first, last):
            m = seen(int(kv), last - first, t - first, mask_block)
            if m == 0:
                out[t], size[t], lse[:, t] = 0.0, 0.0, -np.inf
                continue
            for h in range(hq):
                g = h // (hq // hkv)
                with np.errstate(invalid="ignore", over="ignore"):
                    x = k[:m, g] @ q[t, h].astype(np.float64) * scale
                    top = x.max()
                    p = np.exp(x - top)
                    z = p.sum()
                    out[t, h] = p @ v[:m, g] / z
                    size[t, h] = p @ np.abs(v[:m, g]) / z
                    spread[h, t] = (np.abs(k[:m, g]) @ np.abs(q[t, h].astype(np.float64))).max() * scale
                lse[h, t] = top + math.log(z)
    return out, lse, size, spread
