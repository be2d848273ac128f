"""Inputs whose order hangs on how exactly a selection over beams forms and compares its candidates, and what that order has to be.

A row's cost ln sum_j e^(z_j - m), m its largest logit, may be off by
  E = 2^-23 sum_{z_j < m} p_j (1 + m - z_j):
a term is off by the roundings of z_j - m and of the exponent (2^-24 |z_j - m| each, relative) and by the exponential's 1 ulp, the largest's by nothing;
everything behind the terms is in 64 bits: n additions of 2^-53 of the sum, and a few 2^-53 of a candidate.  Candidates further apart than the E of
both have one order."""
import numpy as np


def bound(z, finished=None):
    """E of every row."""
    z = np.asarray(z, np.float64)
    below = z.max(1, keepdims=True) - z
    with np.errstate(invalid="ignore"):
        p = np.exp(-below)
        e = 2.0 ** -23 * np.where(p > 0, p * (1 + below), 0.0)
    e[below == 0] = 0
    e = e.sum(1) / p.sum(1) + z.shape[1] * 2.0 ** -53
    return e if finished is None else np.where(np.asarray(finished) != 0, 0.0, e)


def misplaced(c, e, beams, parent, token):
    """Pairs of candidates (c[row][token], off by e[row] at most) in an order that cannot be, and how many pairs of neighbours in the true order can have
    one order only."""
    wrong = decided = 0
    n = c.shape[1]
    for g, (p, t) in enumerate(zip(parent, token)):
        part = c[g * beams:(g + 1) * beams]
        slack = np.repeat(e[g * beams:(g + 1) * beams], n) + 2.0 ** -50 * np.abs(np.where(np.isfinite(part), part, 0)).reshape(-1)
        flat, at = part.reshape(-1), (np.asarray(p) - g * beams) * n + np.asarray(t)
        assert (at >= 0).all()
        v, s = flat[at], slack[at]
        for j in range(len(at)):
            wrong += int((v[j] + s[j] < v[j + 1:] - s[j + 1:]).sum())
        rest = np.ones(len(flat), bool)
        rest[at] = False
        if rest.any():
            wrong += int((v + s < (flat[rest] - slack[rest]).max()).sum())
        order = np.argsort(-flat)[:len(at) + 1]
        decided += int((flat[order][:-1] - slack[order][:-1] > flat[order][1:] + slack[order][1:]).sum())
    return wrong, decided


def close_rows(seed, groups, beams, n, around, apart, spread, peak, bf16=False):
    """Logits (fp32, or values of bf16) and scores whose best continuation of every beam stands near `around`: the scores are chosen from the
    costs in 64 bits so that they do, `apart` from each other in a random order, as far as fp32 can hold such scores."""
    rng = np.random.default_rng(seed)
    z = (rng.standard_normal((groups * beams, n)) * spread).astype(np.float32)
    z[np.arange(len(z)), rng.integers(0, n, len(z))] = np.float32(z.max() + peak)
    if bf16:  # (rounded towards zero)
        z = (z.view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)
    x = z.astype(np.float64)
    cost = np.log(np.exp(x - x.max(1, keepdims=True)).sum(1))
    rank = np.concatenate([rng.permutation(beams) for _ in range(groups)])
    return z, (around - apart * rank + cost).astype(np.float32)


# groups, beams, n, scores around, apart, spread, peak, bf16
CLOSE = [(4, 32, 700, -40.0, 1e-6, 1.0, 4.0, False), (4, 32, 4001, -40.0, 1e-6, 1.0, 9.0, False), (3, 32, 5000, -1000.0, 4e-6, 2.0, 3.0, False),
         (3, 32, 33000, -1000.0, 4e-6, 2.5, 2.0, False), (4, 16, 2000, -0.01, 1e-8, 1.0, 14.0, False), (2, 32, 40001, -0.01, 1e-8, 1.0, 18.0, False),
         (3, 32, 9000, -40.0, 1e-6, 1.0, 9.0, True), (2, 32, 66000, -1000.0, 4e-6, 2.0, 3.0, True), (3, 32, 5003, -0.01, 1e-8, 1.0, 16.0, True),
         (1, 4, 700001, -1000.0, 2e-5, 1.0, 12.0, False)]
