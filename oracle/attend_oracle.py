"""Attention of single query rows over their own keys and values in 64 bits: what attention over shared prefixes is checked against."""
from __future__ import annotations

import numpy as np


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray):
    """q [Hq, dh], k and v [n, Hkv, dh] -> (o [Hq, dh], sum of p |v| [Hq, dh]); zeros where n is 0.  Query head h uses K/V head h // (Hq / Hkv)."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    if not len(k):
        return np.zeros_like(q), np.zeros_like(q)
    group = q.shape[0] // k.shape[1]
    k, v = np.repeat(k, group, 1), np.repeat(v, group, 1)
    s = np.einsum("hd,nhd->hn", q, k) / np.sqrt(q.shape[1])
    p = np.exp(s - s.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    return np.einsum("hn,nhd->hd", p, v), np.einsum("hn,nhd->hd", p, np.abs(v))
