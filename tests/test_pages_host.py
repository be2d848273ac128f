"""Without a GPU: the oracle of forking and compacting block tables by hand, and the refusals of the entry points."""
import ctypes as C

import pytest

from oracle import pages_oracle as P
from paper_2506_10470_amd import tdp


def test_beams_of_a_prompt_by_hand():
    # a prompt of 20 tokens in pages 3 and 5 becomes three rows: page 3 is shared, page 5 goes on in the first of them
    t, n, refs, copies, status = P.fork([0, 0, 0], [[3, 5, -1]], [20], [1, 1, 1], [0, 0, 0, 1, 0, 1], 3)
    assert t == [[3, 5, -1], [3, 0, -1], [3, 1, -1]] and n == [21, 21, 21]
    assert refs == [1, 1, 0, 3, 0, 1] and copies == [(-1, -1), (5, 0), (5, 1)] and status == (0, 0, 2, 4)
    # a page that somebody else holds as well is copied by the first row too
    t, _, refs, copies, _ = P.fork([0], [[3, 5]], [20], [12], [0, 1, 0, 1, 0, 2], 2)
    assert t == [[3, 0]] and refs == [1, 1, 0, 1, 0, 1] and copies == [(5, 0)]


def test_release_and_new_rows_by_hand():
    t, n, refs, copies, status = P.fork([-1, 1], [[0], [2]], [16, 16], [17, 0], [1, 0, 1, 0], 2)
    assert t == [[1, 3], [2, -1]] and n == [17, 16] and refs == [0, 1, 1, 1] and copies == [(-1, -1)] * 2 and status == (0, 0, 2, 2)
    assert P.fork([0], [[0]], [16], [17], [1, 0, 1], 3)[4] == (1, 0, 0, 1)      # a page is missing
    assert P.fork([0], [[0]], [16], [17], [1, 0, 1], 2)[4] == 1                 # longer than a row


def test_compaction_by_hand():
    # pages 1, 6 and 7 are in the row, 5 is held by somebody else
    t, refs, moves, status = P.compact([[7, 1, 6, -1]], [40], [0, 1, 0, 0, 0, 1, 1, 1], 3, 4)
    assert t == [[0, 1, 2, -1]] and moves == [(7, 0), (6, 2), (-1, -1)] and refs == [1, 1, 1, 0, 0, 1, 0, 0] and status == (0, 0, 2, 4)
    assert P.compact([[7, 1, 6, -1]], [40], [0, 1, 0, 0, 0, 1, 1, 1], 1, 4)[2] == [(7, 0)]
    assert P.compact([[9]], [1], [0, 1], 1, 1)[3] == (0, 1, 0, 1)


@pytest.mark.parametrize("bad", [dict(num_pages=0), dict(num_pages=(1 << 22) + 1), dict(max_rows=0), dict(max_rows=8193),
                                 dict(max_pages_per_seq=0), dict(max_pages_per_seq=(1 << 16) + 1)])
def test_pages_reject_bad_configurations(bad):
    cfg = dict(num_pages=64, max_rows=4, max_pages_per_seq=4)
    cfg.update(bad)
    with pytest.raises(tdp.TdpError) as e:
        tdp.tdp_pages_create(tdp.PagesConfig(**cfg))
    assert e.value.code == tdp.EINVAL and tdp.last_error()


def test_pages_reject_null_objects():
    h = C.c_void_p()
    assert tdp.lib.tdp_pages_create(None, C.byref(h)) == tdp.EINVAL
    assert tdp.lib.tdp_pages_create(C.byref(tdp.PagesConfig(64, 4, 4)), None) == tdp.EINVAL
    assert tdp.lib.tdp_pages_fork(None, 16, 16, 16, 1, None, 1, 1, 16, 16, 16, 16, 16, 16, None) == tdp.EINVAL
    assert tdp.lib.tdp_pages_compact(None, 16, 16, 1, 1, 16, 16, 16, 16, 16, None) == tdp.EINVAL
    assert tdp.lib.tdp_stage_kv_copy_pages(None, 16, 1, None) == tdp.EINVAL
    tdp.lib.tdp_pages_destroy(None)
