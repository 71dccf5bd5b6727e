"""CPU oracle of sampling from filtered distributions (plain Python / numpy, fp64), written from the definition.

TEST INFRASTRUCTURE ONLY: imported by the tests, never by the product package.

Weights exp((x - max) / T), zero below 2^-1000; order: larger logit first, lower index among equals; kept: the first
top_k of the order, of those the ones before which less than top_p of their weight has come, of those the ones of weight
at least min_p; token: the first kept one in index order whose running weight exceeds uniform * kept weight.
"""
from __future__ import annotations

import math

import numpy as np


def weights(x, T):
    """x: float64 logits without NaN, something above -inf."""
    m = x.max()
    with np.errstate(invalid="ignore"):
        gap = np.where(x == m, 0.0, (x - m) / T)
    return np.where(gap < -1000.0 * math.log(2.0), 0.0, np.exp(np.maximum(gap, -1000.0)))


def kept_set(x, w, top_k=0, top_p=1.0, min_p=0.0):
    """Indices kept, in the order."""
    order = np.lexsort((np.arange(len(x)), -x)).tolist()
    if 0 < top_k < len(x):
        order = order[:top_k]
    if top_p <= 0:
        order = order[:1]
    elif top_p < 1:
        total = math.fsum(w[i] for i in order)
        kept, before = [], 0.0
        for i in order:
            if not before < top_p * total:
                break
            kept.append(i)
            before += w[i]
        order = kept
    if min_p > 0:
        order = [i for i in order if w[i] >= min_p]
    return order


def token(x, u, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    x = np.asarray(x, dtype=np.float64)
    if np.isnan(x).all():
        return 0
    x = np.where(np.isnan(x), -np.inf, x)
    if x.max() == -np.inf:
        raw = np.asarray(x)
        return int(np.flatnonzero(raw == -np.inf)[0])
    if T == 0:
        return int(x.argmax())
    w = weights(x, T)
    kept = [i for i in sorted(kept_set(x, w, top_k, top_p, min_p)) if w[i] > 0]
    total = math.fsum(w[i] for i in kept)
    running = 0.0
    for i in kept:
        running += w[i]
        if u < 1 and running > u * total:                    # (nothing exceeds all of the weight; the rounded sum may)
            return i
    return kept[-1]


def first_above_nan(row):
    """A row of NaNs and -inf only: its first -inf, or 0."""
    at = np.flatnonzero(np.asarray(row) == -np.inf)
    return int(at[0]) if len(at) else 0


def sample(logits, uniform, temperature=None, top_k=None, top_p=None, min_p=None):
    """logits [B, N, V], uniform [B, N] -> int32 [B, N] (parameters [B] or None)."""
    B, N, _ = logits.shape
    at = lambda a, b, d: d if a is None else float(a[b])                                # noqa: E731
    out = np.zeros((B, N), np.int32)
    for b in range(B):
        for r in range(N):
            row = np.asarray(logits[b, r], dtype=np.float64)
            if not (row > -np.inf).any():
                out[b, r] = first_above_nan(row)
            else:
                out[b, r] = token(row, float(uniform[b, r]), at(temperature, b, 1.0), int(at(top_k, b, 0)), at(top_p, b, 1.0), at(min_p, b, 0.0))
    return out
