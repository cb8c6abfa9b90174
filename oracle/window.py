"""Attention under a sliding window with sinks, in float64, one row at a time over the
keys that row sees.

Token i of n new ones sits at position p = kv - n + i, in the mask's block of m
positions that starts at p0 = p // m * m.  It sees the keys t < min(kv, p0 + m) with
t > p0 - window or t < sinks (window 0: all of them; none if p < 0).  A slot of a
verification step sees the cached keys t > prefix - window or t < sinks, and the new
slots that the temporal mask allows."""

from __future__ import annotations

import math

import numpy as np

from .chunk import gather
from .mask import new_slot_visibility, row_valid


def keys(kv: int, n: int, i: int, mask_block: int, window: int, sinks: int) -> list:
    p = kv - n + i
    if p < 0:
        return []
    block = p // mask_block if mask_block else 0
    end = min(kv, (block + 1) * mask_block) if mask_block else kv
    return [t for t in range(end) if not window or t > block * mask_block - window or t < sinks]


def row(q, k, v, scale):
    """(output, log-sum-exp, weighted |v|, largest sum of |q k| scale) of one query."""
    if len(k) == 0:
        return 0.0, -np.inf, 0.0, 0.0
    with np.errstate(invalid="ignore", over="ignore"):
        x = k @ q * scale
        top = x.max()
        p = np.exp(x - top)
        z = p.sum()
        return p @ v / z, top + math.log(z), p @ np.abs(v) / z, (np.abs(k) @ np.abs(q)).max() * scale


def chunk_attention(q, k_cache, v_cache, table, q_starts, kv_lens, *, mask_block=1, window=0, sinks=0, page=0, scale=0.0):
    """(out [tokens, Hq, d], lse [Hq, tokens], weighted |v|, largest sum of |q k| scale
    [Hq, tokens]); rows outside q_starts' range are NaN."""
    T, hq, d = q.shape
    hkv = k_cache.shape[2]
    scale = scale or 1.0 / math.sqrt(d)
    out, size = np.full((T, hq, d), np.nan), np.full((T, hq, d), np.nan)
    lse, spread = np.full((hq, T), np.nan), np.zeros((hq, T))
    for b, kv in enumerate(kv_lens):
        first, last = int(q_starts[b]), int(q_starts[b + 1])
        if first == last:
            continue
        k = gather(k_cache, table, b, int(kv), page).astype(np.float64)
        v = gather(v_cache, table, b, int(kv), page).astype(np.float64)
        for t in range(first, last):
            seen = keys(int(kv), last - first, t - first, mask_block, window, sinks)
            for h in range(hq):
                g = h // (hq // hkv)
                out[t, h], lse[h, t], size[t, h], spread[h, t] = row(q[t, h].astype(np.float64), k[seen, g], v[seen, g], scale)
    return out, lse, size, spread


def verify_attention(q, k_new, v_new, k_cache, v_cache, table, prefix_lens, step_map, num_ref, *, window=0, sinks=0,
                     page=0, scale=0.0):
    """The same of a verification step: q [batch, B + L, Hq, d]; lse and spread [batch, Hq, B + L]."""
    b, n, hq, d = q.shape
    hkv, L = k_new.shape[2], n - step_map.shape[1]
    scale = scale or 1.0 / math.sqrt(d)
    out, size = np.zeros((b, n, hq, d)), np.zeros((b, n, hq, d))
    lse, spread = np.full((b, hq, n), -np.inf), np.zeros((b, hq, n))
    for i in range(b):
        prefix = int(prefix_lens[i])
        old = [t for t in range(prefix) if not window or t > prefix - window or t < sinks]
        k = gather(k_cache, table, i, prefix, page).astype(np.float64)[old]
        v = gather(v_cache, table, i, prefix, page).astype(np.float64)[old]
        allowed, live = (f(step_map[i], int(num_ref[i]), L) for f in (new_slot_visibility, row_valid))
        for s in range(n):
            if not live[s]:
                continue
            new = np.flatnonzero(allowed[s])
            for h in range(hq):
                g = h // (hq // hkv)
                kk = np.concatenate([k[:, g], k_new[i, new, g]])
                vv = np.concatenate([v[:, g], v_new[i, new, g]])
                out[i, s, h], lse[i, h, s], size[i, s, h], spread[i, h, s] = row(q[i, s, h].astype(np.float64), kk, vv, scale)
    return out, lse, size, spread
