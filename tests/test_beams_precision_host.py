"""Without a GPU: the inputs that pin the precision of beam selection do so.  A selection in 64 bits passes their check; one that forms its sums
in fp32, or that compares in fp32, does not."""
import numpy as np
import pytest

from beams_helpers import CLOSE, bound, close_rows, misplaced
from oracle import beams_oracle as B


def ranked(c, beams, n_out):
    """The n_out largest of c by groups, of equal ones the first."""
    n = c.shape[1]
    flat = c.reshape(-1, beams * n)
    order = np.argsort(-flat, axis=1, kind="stable")[:, :n_out]
    return order // n + np.arange(len(flat))[:, None] * beams, order % n


@pytest.mark.parametrize("case", CLOSE)
def test_close_candidates_tell_fp32_from_64_bits(case):
    groups, beams, n, around = case[:4]
    z, scores = close_rows(1, *case)
    c, e, n_out = B.candidates(z, scores, None, -1), bound(z), min(beams, 32)
    parent, token, _, _ = B.select(z, scores, beams, n_out)
    wrong, decided = misplaced(c, e, beams, parent, token)
    assert wrong == 0 and decided >= groups * n_out / 3      # (the order of that many neighbours is settled)
    # sums of fp32 (numpy adds in pairs, which is as exact as fp32 gets), the rest in 64 bits
    m = z.max(1, keepdims=True)
    total = np.exp(z - m).sum(1, keepdims=True)
    assert total.dtype == np.float32
    sums = scores[:, None].astype(np.float64) + ((z.astype(np.float64) - m) - np.log(total.astype(np.float64)))
    # and all of it in fp32
    single = scores[:, None] + ((z - m) - np.log(total))
    assert single.dtype == np.float32
    assert misplaced(c, e, beams, *ranked(single, beams, n_out))[0] > 0
    if around > -1:
        assert misplaced(c, e, beams, *ranked(sums, beams, n_out))[0] > 0


def test_a_row_of_lowest_values_is_an_even_distribution():
    """Each of n tokens at the type's lowest value costs ln n, as n equal tokens do anywhere."""
    for value in (np.finfo(np.float32).min, -1e30, 0.0, 1e30):
        _, token, score, _ = B.select(np.full((1, 3001), value, np.float32), [-2.0], 1, 3)
        assert token.tolist() == [[0, 1, 2]] and np.allclose(score, -2.0 - np.log(3001), rtol=1e-15)
