"""Selection over beams and vocabulary in 64 bits: what tdp_beams_select is checked against."""
from __future__ import annotations

import numpy as np


def candidates(logits: np.ndarray, scores: np.ndarray, finished, end_token: int) -> np.ndarray:
    """c[row][token] for rows of logits, minus infinity where there is no candidate."""
    z = np.asarray(logits, np.float64)
    with np.errstate(all="ignore"):
        top = np.max(z, 1, keepdims=True)                       # (NaN stays)
        # (the logarithm joins the distance to the largest, not the largest: beside -3e38 it would be lost)
        c = np.asarray(scores, np.float64)[:, None] + ((z - top) - np.log(np.exp(z - top).sum(1, keepdims=True)))
    if finished is not None:
        done = np.asarray(finished) != 0
        c[done] = -np.inf
        c[done, end_token] = np.asarray(scores, np.float64)[done]
    c[np.isnan(c)] = -np.inf
    return c


def select(logits, scores, beams: int, n_out: int, finished=None, end_token: int = -1):
    """-> (parent, token, score, finished), each [groups][n_out]"""
    z = np.asarray(logits, np.float64)
    c = candidates(z, scores, finished, end_token)
    groups, n = len(z) // beams, z.shape[1]
    parent, token = np.full((groups, n_out), -1), np.full((groups, n_out), -1)
    score = np.full((groups, n_out), -np.inf)
    for g in range(groups):
        flat = c[g * beams:(g + 1) * beams].reshape(-1)
        tokens = np.tile(np.arange(n), beams)
        order = np.lexsort((tokens, -z[g * beams:(g + 1) * beams].reshape(-1), np.repeat(np.arange(beams), n), -flat))[:n_out]
        order = order[flat[order] > -np.inf]
        parent[g, :len(order)] = g * beams + order // n
        token[g, :len(order)] = order % n
        score[g, :len(order)] = flat[order]
    return parent, token, score, ((token == end_token) & (token >= 0)).astype(int)
