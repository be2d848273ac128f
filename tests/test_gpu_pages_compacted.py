"""A pool that nobody else holds pages of, compacted with as many moves as there are pages: what is in use stands at its front without a gap."""
import random

import pytest
import torch

from oracle import pages_oracle as P
from paper_2506_10470_amd import tdp
from stage_helpers import i32
from test_gpu_pages import Pages, pool_of_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_rows,width,count,longest,moves,in_place", [
    (1, 4, 16, 60, 16, False), (3, 8, 64, 100, 64, True), (40, 12, 900, 180, 900, False), (40, 12, 900, 180, 1000, True), (7, 3, 4097, 48, 4097, False),
    (300, 20, 9001, 300, 9001, False), (70, 70, 20000, 1000, 20000, True), (2, 9, 40, 100, 400, True), (2000, 6, 65536, 96, 65536, False)])
def test_pages_in_use_stand_at_the_front(n_rows, width, count, longest, moves, in_place):
    rng = random.Random(3 * n_rows + count)
    lens = [rng.randint(1, longest) for _ in range(n_rows)]
    tables, refs = pool_of_rows(rng, n_rows, width, count, lens, pins=0)
    used = sum(x > 0 for x in refs)
    assert sum(refs) == sum(map(P.pages_of, lens)) and 0 in refs[:max(p for p in range(count) if refs[p])]      # (free ids between used ones)
    with Pages(count, n_rows, width) as pages:
        t, n, r = i32(tables), i32(lens), i32(refs)
        t_out = t if in_place else torch.full_like(t, -9)
        r_out = r if in_place else torch.full_like(r, -9)
        m = torch.full((moves, 2), -9, dtype=torch.int32, device="cuda")
        status = torch.full((4,), -9, dtype=torch.int32, device="cuda")
        tdp.tdp_pages_compact(pages.h, t, n, n_rows, moves, r, r_out, t_out, m, status)
        torch.cuda.synchronize()
        got_refs, got_tables = r_out.tolist(), t_out.tolist()
        assert all(x > 0 for x in got_refs[:used]) and not any(got_refs[used:])
        assert sorted(x for x in got_refs if x) == sorted(x for x in refs if x)
        # the tables name the same pages by their new ids, one to one
        moved = {}
        for old, new, length in zip(tables, got_tables, lens):
            held = P.pages_of(length)
            assert new[held:] == [-1] * (width - held)
            for a, b in zip(old[:held], new[:held]):
                assert moved.setdefault(a, b) == b and 0 <= b < used and got_refs[b] == refs[a]
        assert len(set(moved.values())) == len(moved) == used
        pairs = [(a, b) for a, b in m.tolist() if a >= 0]
        assert dict(pairs) == {a: b for a, b in moved.items() if a != b} and status.tolist() == [0, 0, len(pairs), used]
        assert (got_tables, got_refs, [tuple(x) for x in m.tolist()], tuple(status.tolist())) == P.compact(tables, lens, refs, moves, width)
        # and there is nothing left to move
        again = torch.full((moves, 2), -9, dtype=torch.int32, device="cuda")
        tdp.tdp_pages_compact(pages.h, t_out, n, n_rows, moves, r_out, r_out, t_out, again, status)
        torch.cuda.synchronize()
        assert (again == -1).all() and status.tolist() == [0, 0, 0, used] and t_out.tolist() == got_tables and r_out.tolist() == got_refs
