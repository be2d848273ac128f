"""Without a GPU: the oracle of beam selection by hand, and the refusals of its entry points."""
import ctypes as C

import numpy as np
import pytest

from oracle import beams_oracle as B
from paper_2506_10470_amd import tdp

INF = float("inf")


def test_two_beams_by_hand():
    z = np.log([[0.5, 0.25, 0.25], [0.1, 0.8, 0.1]])
    parent, token, score, fin = B.select(z, [0.0, np.log(0.5)], 2, 4, None, 1)
    assert parent.tolist() == [[0, 1, 0, 0]] and token.tolist() == [[0, 1, 1, 2]] and fin.tolist() == [[0, 1, 1, 0]]
    assert np.allclose(score, np.log([[0.5, 0.4, 0.25, 0.25]]))
    parent, token, score, fin = B.select(z, [0.0, np.log(0.5)], 2, 3, [1, 0], 2)     # the first beam is finished
    assert parent.tolist() == [[0, 1, 1]] and token.tolist() == [[2, 1, 0]] and fin.tolist() == [[1, 0, 0]]
    assert np.allclose(score, np.log([[1, 0.4, 0.05]]))


def test_places_without_a_candidate():
    z = np.array([[0, -INF, 0], [np.nan, 0, 0], [INF, 0, 0], [-INF] * 3])
    parent, token, score, _ = B.select(z, [0.0] * 4, 4, 3)
    assert parent.tolist() == [[0, 0, -1]] and token.tolist() == [[0, 2, -1]] and np.allclose(score[0, :2], np.log(0.5)) and score[0, 2] == -INF
    assert B.select(np.zeros((1, 2)), [-INF], 1, 2)[0].tolist() == [[-1, -1]]


@pytest.mark.parametrize("bad", [dict(max_rows=0), dict(max_rows=(1 << 16) + 1), dict(max_out=0), dict(max_out=33)])
def test_beams_reject_bad_configurations(bad):
    cfg = dict(max_rows=8, max_out=8)
    cfg.update(bad)
    with pytest.raises(tdp.TdpError) as e:
        tdp.tdp_beams_create(tdp.BeamsConfig(**cfg))
    assert e.value.code == tdp.EINVAL and tdp.last_error()


def test_beams_reject_null_objects():
    h = C.c_void_p()
    assert tdp.lib.tdp_beams_create(None, C.byref(h)) == tdp.EINVAL
    assert tdp.lib.tdp_beams_create(C.byref(tdp.BeamsConfig(8, 8)), None) == tdp.EINVAL
    assert tdp.lib.tdp_beams_select(None, 16, 0, 1, 1, 8, 8, 16, None, -1, 1, 16, 16, 16, None, None) == tdp.EINVAL
    tdp.lib.tdp_beams_destroy(None)
