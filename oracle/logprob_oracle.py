"""CPU oracle for log-probabilities of rows of logits, in fp64.

TEST INFRASTRUCTURE ONLY: imported by tests, never by the product path; shares no code with the HIP kernels.
"""
from __future__ import annotations

import numpy as np


def row_answer(z: np.ndarray, target, n_top: int):
    """(logprob of the target, entropy, indices, their log-probabilities) of one row.  target None: the row's largest logit; outside
    the row: minus infinity.  Indices: by logit, of equal ones the lower first, NaN left out, -1 behind the last."""
    z = np.asarray(z, dtype=np.float64)
    numbers = np.flatnonzero(~np.isnan(z))
    order = numbers[np.lexsort((numbers, -z[numbers]))][:n_top]
    index = np.full(n_top, -1, dtype=np.int64)
    index[:len(order)] = order
    if np.isnan(z).any() or np.isposinf(z).any() or not np.isfinite(z).any():
        inside = target is None or 0 <= target < len(z)
        return (np.nan if inside else -np.inf), np.nan, index, np.full(n_top, np.nan)
    m = z.max()
    p = np.exp(z - m)
    log_p = z - m - np.log(p.sum())
    p = p / p.sum()
    entropy = -np.sum(p[p > 0] * log_p[p > 0])
    logprob = log_p.max() if target is None else log_p[target] if 0 <= target < len(z) else -np.inf
    return logprob, entropy, index, log_p[order]


def answer(z: np.ndarray, targets, n_top: int):
    """row_answer of every row, as four arrays."""
    rows = [row_answer(r, None if targets is None else int(targets[i]), n_top) for i, r in enumerate(np.asarray(z))]
    return (np.array([r[0] for r in rows]), np.array([r[1] for r in rows]), np.array([r[2] for r in rows]).reshape(len(rows), n_top),
            np.array([r[3] for r in rows]).reshape(len(rows), n_top))


def tolerance(z: np.ndarray, links=None):
    """(of a log-probability, of an entropy) per row: what an fp32 evaluation relative to the row's maximum can be off by.

    With u = 2^-24, d = z - m (spread R = max |d| over what e^d does not turn into 0 in fp32, at most 104), D = sum p |d|:
    a difference is off by u |d|, the product with log2 e in front of the exponential by u |d| of its result, the exponential by 2 u:
    (2 |d| + 2) u per term, (2 D + 2) u of s.  Moving a partial sum to a larger maximum: (2 |change| + 3) u, the changes of a chain add up
    to R, in `links` links: 6 + 4 exchanges and the turns of a thread that raise its maximum, of 32768 logits or more, or of 16384 of a
    projection in pieces; up to 14 of those, a row of 229376, it is 24 links and (2 R + 72) u, beyond that as many more as a row
    that rises from turn to turn has.  (A row known to rise less often may give its own number.)
    Additions: up to 200 u.  A row's are 64 in a turn, 2 u for the sum of the turns, which is kept in two numbers, and 10 exchanges; a
    projection's 34, one for 16384 columns (of 2 million: 128) and 10.  ln s: off by that sum (relative error of s) and 2 u |ln s| of its own.
    t = sum e^d d: the same per term and 2 u more, weighted with |d| <= R: (2 R + 4) u D, and the chain's and the additions' share of D."""
    u = 2.0 ** -24
    out = []
    for r in np.asarray(z, dtype=np.float64):
        chain = 3 * (links or 10 + max(14, -(-len(r) // 16384)))
        r = r[np.isfinite(r)]
        if not len(r):
            out.append((0.0, 0.0))
            continue
        d = r - r.max()
        e = np.exp(d)
        D = np.sum(e * -d) / e.sum()
        R = min(104.0, -d.min())
        s = (2 * D + 2 + 2 * R + chain + 200 + 2 * abs(np.log(e.sum()))) * u
        out.append((s, s + (2 * R + 4) * D * u + (2 * R + chain + 200 + 4) * D * u + 2 * u * D))
    return np.array(out).reshape(-1, 2).T
