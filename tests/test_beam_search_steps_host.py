"""Without a GPU: under the weights that the steps of a search are checked with, a fault of the kind that forked tables and shared prefixes can
have moves the logits far beyond the tolerance of that check.  The faults are planted in the oracle."""
import numpy as np
import pytest

from harness import workload as W
from search_helpers import LOGITS_TOL, LOGITS_TOL_8BIT, SEARCHES, VOCAB, AttentiveOracle
from stage_helpers import row_rel_err


@pytest.mark.parametrize("shape,lengths,beams,max_new,end,kv_scales", SEARCHES)
def test_faults_of_pages_and_prefixes_move_the_logits(shape, lengths, beams, max_new, end, kv_scales):
    tol = LOGITS_TOL if kv_scales is None else LOGITS_TOL_8BIT
    n = max(lengths) + max_new - 1
    model = AttentiveOracle(W.SHAPES[shape], kv_scales)
    tokens, others = (W.token_ids(VOCAB, n, 900 + i).tolist() for i in range(2))
    own, other = model.caches(tokens[:-1]), model.caches(others[:-1])
    want = model.logits(tokens[-1], own)

    def moved(caches):
        return row_rel_err(model.logits(tokens[-1], caches)[None], want[None])

    def foreign(which):         # the keys and values of another beam at these positions
        return moved([(np.where(which[:, None, None], k2, k), np.where(which[:, None, None], v2, v)) for (k, v), (k2, v2) in zip(own, other)])

    at = np.arange(n - 1)
    assert moved([(k[:0], v[:0]) for k, v in own]) > 8 * tol                                        # attention dropped
    assert all(foreign(at // 16 == page) > 4 * tol for page in range((n - 1) // 16))                # a whole page of another beam
    assert foreign(at >= n - 1 - min(3, n - 1)) > 2 * tol                                           # a last page that was not copied
    assert moved([(k[:-1], v[:-1]) for k, v in own]) > (2 if kv_scales is None else 1.25) * tol     # a token less, the position before
    if n > 32:
        assert moved([(k[16:], v[16:]) for k, v in own]) > 4 * tol                                  # a page of the prefix left out
