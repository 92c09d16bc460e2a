"""Attention over a prompt's tokens in float64: causal or not, grouped heads, the log-sum-exp beside the output.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).
"""
from __future__ import annotations

import numpy as np


def prompt_attention(q, k, v, sm_scale, causal=True):
    """q [n_q, Hq, D] (the last n_q of n_k tokens), k, v [n_k, Hkv, D] -> (out [n_q, Hq, D], lse [n_q, Hq]).
    Token i sees keys j <= i + n_k - n_q (causal) or all; one that sees none gets zeros and -inf."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    n_q, hq, d = q.shape
    n_k, hkv, _ = k.shape
    out, lse = np.zeros((n_q, hq, d)), np.full((n_q, hq), -np.inf)
    for i in range(n_q):
        n = min(n_k, max(0, i + n_k - n_q + 1)) if causal else n_k
        if n == 0:
            continue
        for h in range(hkv):
            g = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            s = (q[i, g] @ k[:n, h].T) * float(sm_scale)
            m = s.max(axis=1, keepdims=True)
            w = np.exp(s - m)
            t = w.sum(axis=1, keepdims=True)
            out[i, g] = (w / t) @ v[:n, h]
            lse[i, g] = (m + np.log(t))[:, 0]
    return out, lse
