"""Norm per head and position rotation of queries and keys in float64.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).
"""
from __future__ import annotations

import numpy as np


def norm_rope(x, positions, inv_freq, *, norm=False, weight=None, eps=1e-6, interleaved=False):
    """x [T, H, D], positions [T], or [T, R/2] one for every frequency -> (rotated rows, |a| + |b| of every channel's pair before the rotation: what rounding
    errors are relative to); a row is normed over its D channels, then its first 2 len(inv_freq) channels turn."""
    x = np.asarray(x, np.float64)
    if norm:
        x = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
        if weight is not None:
            x = x * np.asarray(weight, np.float64)
    y, size = x.copy(), np.abs(x)
    half = 0 if inv_freq is None else len(inv_freq)
    if half:
        at = np.asarray(positions, np.float64)
        t = (at[:, None] if at.ndim == 1 else at) * np.asarray(inv_freq, np.float64)[None, :]
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            c, s = np.cos(t[:, i])[:, None], np.sin(t[:, i])[:, None]
            y[..., a] = x[..., a] * c - x[..., b] * s
            y[..., b] = x[..., b] * c + x[..., a] * s
            size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y, size
