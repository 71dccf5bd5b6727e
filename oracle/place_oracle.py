"""CPU oracle of the norm + rotary + cache append step (numpy, fp64).

TEST INFRASTRUCTURE ONLY: imported by the tests, never by the product package.

Per query and key head x of D features: y = x / sqrt(mean(x^2) + eps) * (w + offset); the first rot_dim features are
rotated pair by pair by pos * f_i (pairs (i, i + rot_dim/2) or (2i, 2i + 1)), cosine and sine times `magnitude`.
"""
from __future__ import annotations

import math

import numpy as np


def frequencies(rot_dim, base=10000.0, scaling="plain", factor=1.0, low=1.0, high=4.0, orig_len=0.0):
    f = np.array([base ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)], dtype=np.float64)
    if scaling == "linear":
        return f / factor
    if scaling == "parts":
        out = []
        for x in f:
            turns = orig_len * x / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - low) / (high - low)))
            out.append(x * (keep + (1 - keep) / factor))
        return np.array(out)
    return f


def heads(x, pos, weight=None, norm=True, eps=1e-6, offset=0.0, rot_dim=None, interleaved=False, magnitude=1.0, **freq):
    """x [..., H, D] at position ids pos [...] -> float64 of x's shape."""
    x = np.array(x, dtype=np.float64)
    D = x.shape[-1]
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if weight is not None:
            x = x * (np.asarray(weight, dtype=np.float64) + offset)
    rot = D if rot_dim is None else rot_dim
    out = x.copy()
    f = frequencies(rot, **freq) if rot else []
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        ang = np.asarray(pos, dtype=np.float64)[..., None] * f[i]
        c, s = np.cos(ang) * magnitude, np.sin(ang) * magnitude
        out[..., a] = x[..., a] * c - x[..., b] * s
        out[..., b] = x[..., b] * c + x[..., a] * s
    return out
