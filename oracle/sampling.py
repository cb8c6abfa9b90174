"""Sampling from filtered logits in float64, one row at a time, by sorting: the
tokens in the order of falling logits (lowest index first among equal ones), the
leading parts that top-k, top-p and min-p keep, and the first kept token at which
the running weight exceeds u times the weight of all kept ones."""

from __future__ import annotations

import math

import numpy as np


def sample_row(x: np.ndarray, u: float, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """x [V] float64 -> (token, probability, kept)."""
    x = np.where(np.isnan(x), -np.inf, x) + 0.0            # -0 + 0 == +0
    order = np.argsort(-x, kind="stable")
    top = x[order[0]]
    if top == -math.inf:
        return -1, 0.0, 0
    if not temperature > 0:
        return int(order[0]), 1.0, 1
    with np.errstate(invalid="ignore"):
        gap = np.where(x[order] == top, 0.0, x[order] - top)
    n = int((gap >= -700.0 * temperature).sum())
    w = np.exp(gap[:n] / temperature)
    if top_k > 0:
        w = w[:top_k]
    run = np.cumsum(w)
    n = len(w)
    if top_p < 1.0:
        n = min(n, 1 + int((run < max(top_p, 0.0) * run[-1]).sum()))
    if min_p > 0.0:
        n = min(n, int((w >= min(min_p, 1.0)).sum()))
    at = int((run[:n] <= u * run[n - 1]).sum())
    return int(order[at]), float(w[at] / run[n - 1]), n


def sample(logits, uniforms, temperature, top_k, top_p, min_p):
    """Rows of sample_row; each parameter one number or one a row."""
    rows = len(logits)
    par = [np.broadcast_to(np.asarray(p), (rows,)) for p in (temperature, top_k, top_p, min_p)]
    got = [sample_row(logits[i], float(uniforms[i]), float(par[0][i]), int(par[1][i]),
                      float(par[2][i]), float(par[3][i])) for i in range(rows)]
    return (np.array([g[0] for g in got], np.int32), np.array([g[1] for g in got]),
            np.array([g[2] for g in got], np.int32))
