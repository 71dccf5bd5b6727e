"""CPU oracle of tree attention with capped and distance-biased scores (numpy, fp64).

TEST INFRASTRUCTURE ONLY: imported by the tests, never by the product package.

s = scale q.k of a visible key; s := cap tanh(s / cap); s := s - slope_h (pos_row - pos_key), where context row j is at
position j and tree row c at pos[c]; softmax over the visible keys.
"""
from __future__ import annotations

import numpy as np

from .paged_oracle import visibility


def tree_attention(q, k_cache, v_cache, kv_len, parent, cap=0.0, slopes=None, pos=None, scale=None, spread=False):
    """q [B, N, Hq, D]; caches [B, Hkv, rows, D]; returns float64 [B, N, Hq, D] (rows of illegal sequences are zero);
    with ``spread`` also the weighted sums of |v|, of the same shape."""
    q = np.asarray(q, dtype=np.float64)
    B, N, Hq, D = q.shape
    Hkv, room = k_cache.shape[1], k_cache.shape[2]
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    out, size = np.zeros_like(q), np.zeros_like(q)
    for b in range(B):
        L, par = int(kv_len[b]), np.asarray(parent[b])
        if L < 0 or L + N > room or any(int(par[r]) < -1 or int(par[r]) >= r for r in range(N)):
            continue
        vis = visibility(par, L)
        if slopes is not None:
            at = np.concatenate([np.arange(L), pos[b]]).astype(np.float64)
            away = np.asarray(pos[b], dtype=np.float64)[:, None] - at[None]
        for h in range(Hq):
            kv = h // (Hq // Hkv)
            K = np.asarray(k_cache[b, kv, :L + N], dtype=np.float64)
            V = np.asarray(v_cache[b, kv, :L + N], dtype=np.float64)
            s = scale * (q[b, :, h] @ K.T)
            if cap:
                s = cap * np.tanh(s / cap)
            if slopes is not None:
                s = s - float(slopes[h]) * away
            s = np.where(vis, s, -np.inf)
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            out[b, :, h], size[b, :, h] = p @ V, p @ np.abs(V)
    return (out, size) if spread else out
