"""Forking and compacting block tables and copying pages on the GPU, against the oracle: every number has to be equal."""
import random

import numpy as np
import pytest
import torch

from harness import workload as W
from oracle import pages_oracle as P
from paper_2506_10470_amd import tdp
from stage_helpers import Stage, i32

pytestmark = pytest.mark.gpu
PAGE = 16


class Pages:
    def __init__(self, num_pages, max_rows, width):
        self.h, self.n, self.width = tdp.tdp_pages_create(tdp.PagesConfig(num_pages, max_rows, width)), num_pages, width

    def __enter__(self):
        return self

    def __exit__(self, *a):
        tdp.tdp_pages_destroy(self.h)

    def fork(self, parents, tables, lens, add, refs, n_dst=None, in_place=False, stream=None):
        n_dst = len(parents) if n_dst is None else n_dst
        par = None if parents is None else i32(parents)
        r_in = i32(refs)
        r_out = r_in if in_place else torch.full((self.n,), -7, dtype=torch.int32, device="cuda")
        t = torch.full((max(1, n_dst), self.width), -9, dtype=torch.int32, device="cuda")
        n = torch.full((max(1, n_dst),), -9, dtype=torch.int32, device="cuda")
        copies = torch.full((max(1, n_dst), 2), -9, dtype=torch.int32, device="cuda")
        status = torch.full((4,), -9, dtype=torch.int32, device="cuda")
        each = isinstance(add, (list, tuple))
        tdp.tdp_pages_fork(self.h, par, i32(tables) if len(lens) else None, i32(lens) if len(lens) else None, len(lens),
                           i32(add) if each else None, 0 if each else add, n_dst, r_in, r_out, t, n, copies, status, stream)
        torch.cuda.synchronize()
        return t[:n_dst].tolist(), n[:n_dst].tolist(), r_out.tolist(), [tuple(c) for c in copies[:n_dst].tolist()], tuple(status.tolist())


def pool_of_rows(rng, n_rows, width, count, lens, shared_with_first=0.5, pins=0.1):
    """Tables of n_rows rows of the given lengths over `count` pages, some beginning as the first one does; pages held by others."""
    ids = rng.sample(range(count), count)
    refs, tables = [0] * count, []
    for r, n in enumerate(lens):
        held = P.pages_of(n)
        common = min(n // PAGE, lens[0] // PAGE) if r and rng.random() < shared_with_first else 0
        row = (tables[0][:common] if r else []) + [ids.pop() for _ in range(held - common)]
        for p in row:
            refs[p] += 1
        tables.append(row + [-1] * (width - held))
    for row, n in zip(tables, lens):
        for p in row[:P.pages_of(n)]:
            if rng.random() < pins:
                refs[p] += 1
    for _ in range(min(len(ids) // 4, int(pins * 20))):
        refs[ids.pop()] += 1
    return tables, refs


@pytest.mark.parametrize("n_src,n_dst,width,count,longest,in_place", [
    (1, 4, 8, 64, 100, False), (4, 4, 8, 64, 100, True), (3, 7, 5, 100, 70, False), (16, 16, 33, 700, 500, True), (64, 64, 7, 5000, 100, False),
    (200, 300, 12, 4096, 150, False), (130, 1500, 9, 12289, 100, True), (1025, 1025, 4, 9000, 50, False), (8, 3, 300, 70001, 4700, True)])
def test_forks_of_random_tables(n_src, n_dst, width, count, longest, in_place):
    rng = random.Random(n_src * 1000 + n_dst)
    lens = [rng.randint(0, longest) for _ in range(n_src)]
    lens[-1] = longest // PAGE * PAGE
    lens[0] = longest
    tables, refs = pool_of_rows(rng, n_src, width, count, lens)
    parents = [rng.randrange(-1, n_src) if rng.random() < 0.2 else rng.randrange((n_src + 1) // 2) for _ in range(n_dst)]
    most = width * PAGE
    add = [rng.choice([0, 1, 1, 16, 17]) for _ in parents]
    add = [min(a, most - (lens[p] if p >= 0 else 0)) for a, p in zip(add, parents)]
    want = P.fork(parents, tables, lens, add, refs, width)
    assert want[0] is not None and sum(c[0] >= 0 for c in want[3]) > 0
    with Pages(count, max(n_src, n_dst), width) as pages:
        got = pages.fork(parents, tables, lens, add, refs, in_place=in_place)
        assert got == (want[0], want[1], want[2], want[3], want[4])
        assert min(got[2]) >= 0


def test_rows_go_on_where_no_parents_are_given():
    rng = random.Random(5)
    lens = [33, 32, 1, 0]
    tables, refs = pool_of_rows(rng, 4, 6, 64, lens, 0, 0)
    with Pages(64, 8, 6) as pages:
        want = P.fork([0, 1, 2, 3, -1, -1], tables, lens, [1] * 6, refs, 6)
        assert pages.fork(None, tables, lens, 1, refs, n_dst=6) == want
        want = P.fork([0, 1], tables, lens, [0] * 2, refs, 6)                      # the rest is released
        assert pages.fork(None, tables, lens, 0, refs, n_dst=2) == want


def test_all_rows_released_and_rows_made_from_nothing():
    rng = random.Random(6)
    lens = [70, 70, 5]
    tables, refs = pool_of_rows(rng, 3, 6, 64, lens, 1, 0)
    with Pages(64, 8, 6) as pages:
        got = pages.fork([], tables, lens, 0, refs)
        assert got[2] == [0] * 64 and got[4] == (0, 0, 0, refs.count(0))
        got = pages.fork([-1, -1, -1], [], [], [96, 0, 17], [0] * 64)
        assert got[0] == [[0, 1, 2, 3, 4, 5], [-1] * 6, [6, 7, -1, -1, -1, -1]] and got[1] == [96, 0, 17]
        assert got[2] == [1] * 8 + [0] * 56 and got[4] == (0, 0, 8, 64)
        assert pages.fork([], [], [], 0, refs)[2:] == (refs, [], (0, 0, 0, refs.count(0)))


def test_a_long_row_of_fresh_pages_over_many_chunks():
    rng = random.Random(7)
    count, width = 300_000, 65536
    refs = [1 if rng.random() < 0.7 else 0 for _ in range(count)]
    refs[4096:4 * 4096] = [1] * (3 * 4096)
    want = P.fork([-1, -1], [], [], [width * PAGE, 16 * 5000 + 1], refs, width)
    with Pages(count, 2, width) as pages:
        assert pages.fork([-1, -1], [], [], [width * PAGE, 16 * 5000 + 1], refs) == want


@pytest.mark.parametrize("in_place", [False, True])
def test_nothing_happens_where_a_page_is_missing_or_a_row_is_refused(in_place):
    tables, lens, width = [[3, 5, -1], [0, 1, 2]], [20, 48], 3
    refs = [1, 1, 1, 1, 0, 1]
    left = [[-9] * 3] * 2, [-9] * 2, refs, [(-1, -1)] * 2
    with Pages(6, 4, width) as pages:
        def fork(parents, add, lens=lens, tables=tables):
            return pages.fork(parents, tables, lens, add, refs, in_place=in_place)
        assert fork([0, 0], [1, 13]) == (*left, (1, 0, 0, 1))          # the second row needs two
        assert fork([0, 2], [1, 1])[4][1] == 1                          # no such parent
        assert fork([0, -2], [1, 1])[:4] == left
        assert fork([1, 0], [1, 1])[4][1] == 1                          # longer than a table row
        assert fork([0, 1], [-1, 0])[:4] == left
        assert fork([0, 0], [1, 1], lens=[20, 49])[4][1] == 1           # a released row that cannot be
        assert fork([0, 0], [1, 1], lens=[-1, 0])[4][1] == 2
        assert fork([0, 0], [1, 1], tables=[[3, 6, -1], [0, 1, 2]])[4][1] == 2     # the last page lies outside
        assert fork([0, 0], [1, 1], tables=[[3, -1, -1], [0, 1, 2]])[:4] == left
        got = fork([0, 0], [1, 12])                                     # and with the page that there is, all goes well
        assert got == P.fork([0, 0], tables, lens, [1, 12], refs, width) and got[4] == (0, 0, 1, 1)


@pytest.mark.parametrize("n_rows,width,count,longest,moves,in_place", [
    (1, 4, 16, 60, 16, False), (3, 8, 64, 100, 5, True), (40, 12, 900, 180, 900, False), (40, 12, 900, 180, 37, True),
    (300, 20, 9001, 300, 9001, False), (2, 9, 40, 100, 400, True), (70, 70, 20000, 1000, 1000, True), (5, 2, 5, 16, 5, False)])
def test_compaction_of_random_tables(n_rows, width, count, longest, moves, in_place):
    rng = random.Random(n_rows + count)
    lens = [rng.randint(0, longest) for _ in range(n_rows)]
    tables, refs = pool_of_rows(rng, n_rows, width, count, lens)
    want = P.compact(tables, lens, refs, moves, width)
    with Pages(count, n_rows, width) as pages:
        t, n, r = i32(tables), i32(lens), i32(refs)
        t_out = t if in_place else torch.full_like(t, -9)
        r_out = r if in_place else torch.full_like(r, -9)
        m = torch.full((moves, 2), -9, dtype=torch.int32, device="cuda")
        status = torch.full((4,), -9, dtype=torch.int32, device="cuda")
        tdp.tdp_pages_compact(pages.h, t, n, n_rows, moves, r, r_out, t_out, m, status)
        torch.cuda.synchronize()
        got = t_out.tolist(), r_out.tolist(), [tuple(x) for x in m.tolist()], tuple(status.tolist())
        assert got == want
        if moves >= count and not any(a != b for a, b in zip(refs, np.bincount([p for row, k in zip(tables, lens) for p in row[:P.pages_of(k)]],
                                                                                minlength=count))):
            assert got[1].index(0) == sum(x > 0 for x in refs)


def test_compaction_moves_nothing_where_a_row_is_refused():
    """And the call behind that is what it would have been."""
    tables, lens, refs = [[7, 9, -1], [6, -1, -1]], [20, 3], [0] * 6 + [1, 1]
    good = [[7, 6, -1], [6, -1, -1]], [20, 3], [0] * 6 + [2, 1]
    with Pages(8, 4, 3) as pages:
        for lens, tables in ((lens, tables), ([49, 3], [[7, 5, 4], [6, -1, -1]]), ([-1, 3], [[7, 5, 4], [6, -1, -1]])):
            t, r = i32(tables), torch.empty(8, dtype=torch.int32, device="cuda")
            out, m, status = torch.empty_like(t), torch.empty((8, 2), dtype=torch.int32, device="cuda"), i32([9] * 4)
            tdp.tdp_pages_compact(pages.h, t, i32(lens), 2, 8, i32(refs), r, out, m, status)
            assert status.tolist() == [0, 1, 0, 2] and (m == -1).all() and r.tolist() == refs
            assert out.tolist() == P.compact(tables, lens, refs, 8, 3)[0]
            t = i32(good[0])
            tdp.tdp_pages_compact(pages.h, t, i32(good[1]), 2, 8, i32(good[2]), r, out, m, status)
            assert (out.tolist(), r.tolist(), [tuple(x) for x in m.tolist()], tuple(status.tolist())) == P.compact(*good, 8, 3)
            assert status.tolist() == [0, 0, 2, 2]


@pytest.mark.parametrize("shape,kv_scales", [("tiny", None), ("tiny_gqa", (0.5, 0.25)), ("tiny_h128", None), ("tiny_mqa", (1.0, 1.0)), ("13b_quarter", None)])
def test_pages_are_copied_in_every_layer_and_nowhere_else(shape, kv_scales):
    sh = W.SHAPES[shape].with_layers(3)
    if sh.d_model > 1000:       # (the projections are not what is tested)
        sh = W.StageShape("wide_cache", 3, 64, sh.n_q_heads, sh.n_kv_heads, sh.head_dim, 64)
    count = 41
    with Stage(tdp, sh, count, 2, 0, 0, 4, load_weights=False, kv_scales=kv_scales) as st:
        want = []
        for l in range(3):
            for t in st.raw_pools(l):
                raw = t.view(torch.uint8)
                raw.copy_(torch.randint(0, 256, raw.shape, dtype=torch.uint8, device="cuda"))
                want.append(raw.clone().view(count, -1))
        pairs = [(3, 40), (-1, -1), (5, 0), (3, 7), (-1, 9), (8, -1), (41, 10), (11, 41), (12, 13)]
        for w in want:
            for a, b in [(3, 40), (5, 0), (3, 7), (12, 13)]:
                w[b] = w[a]
        tdp.tdp_stage_kv_copy_pages(st.h, i32(pairs), len(pairs))
        tdp.tdp_stage_kv_copy_pages(st.h, None, 0)
        torch.cuda.synchronize()
        got = [t.view(torch.uint8).view(count, -1) for l in range(3) for t in st.raw_pools(l)]
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        with pytest.raises(tdp.TdpError):
            tdp.tdp_stage_kv_copy_pages(st.h, None, 1)
        with pytest.raises(tdp.TdpError):
            tdp.tdp_stage_kv_copy_pages(st.h, i32(pairs), -1)


def test_refusals():
    with Pages(64, 4, 4) as pages:
        t, n, r, c, s = i32(np.zeros((4, 4))), i32([0] * 4), i32([0] * 64), i32(np.zeros((4, 2))), i32([0] * 4)
        t2, n2, r2 = t.clone(), n.clone(), r.clone()
        ok = dict(parents=None, st=t, sl=n, n_src=4, add=None, add_all=1, n_dst=4, ri=r, ro=r2, dt=t2, dl=n2, c=c, s=s)
        for bad in [dict(n_src=5), dict(n_dst=5), dict(n_src=-1), dict(n_dst=-1), dict(add_all=-1), dict(ri=None), dict(ro=None), dict(s=None),
                    dict(st=None), dict(sl=None), dict(dt=None), dict(dl=None), dict(c=None), dict(dt=t), dict(dl=n), dict(dt=t[2:], n_dst=2),
                    dict(ro=r.data_ptr() + 4)]:
            a = {**ok, **bad}
            with pytest.raises(tdp.TdpError) as e:
                tdp.tdp_pages_fork(pages.h, a["parents"], a["st"], a["sl"], a["n_src"], a["add"], a["add_all"], a["n_dst"], a["ri"], a["ro"], a["dt"],
                                   a["dl"], a["c"], a["s"])
            assert e.value.code == tdp.EINVAL, bad
        m = i32(np.zeros((64, 2)))
        ok = dict(st=t, sl=n, n=4, moves=64, ri=r, ro=r2, dt=t2, m=m, s=s)
        for bad in [dict(n=5), dict(n=-1), dict(moves=0), dict(moves=(1 << 22) + 1), dict(ri=None), dict(ro=None), dict(m=None), dict(s=None), dict(st=None),
                    dict(sl=None), dict(dt=None), dict(dt=t[2:], n=3), dict(ro=r.data_ptr() + 4)]:
            a = {**ok, **bad}
            with pytest.raises(tdp.TdpError) as e:
                tdp.tdp_pages_compact(pages.h, a["st"], a["sl"], a["n"], a["moves"], a["ri"], a["ro"], a["dt"], a["m"], a["s"])
            assert e.value.code == tdp.EINVAL, bad


def test_steps_on_a_side_stream_and_in_a_graph():
    """A chain of beam steps between two sets of tables, captured once and replayed with new parents, gives what the oracle gives."""
    width, count, rows = 8, 256, 6
    rng = random.Random(11)
    with Pages(count, rows, width) as pages:
        tables, lens, refs = [[-1] * width] * rows, [0] * rows, [0] * count
        a = dict(t=i32(tables), n=i32(lens), r=i32(refs))
        b = {k: torch.empty_like(v) for k, v in a.items()}
        par = i32([-1] * rows)
        copies, status = torch.empty((rows, 2), dtype=torch.int32, device="cuda"), torch.empty(4, dtype=torch.int32, device="cuda")

        def step(x, y, stream):
            tdp.tdp_pages_fork(pages.h, par, x["t"], x["n"], rows, None, 1, rows, x["r"], y["r"], y["t"], y["n"], copies, status, stream)

        graph = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        step(a, b, side)                 # (the kernels are loaded)
        torch.cuda.synchronize()
        a["t"].copy_(i32(tables)), a["n"].copy_(i32(lens)), a["r"].copy_(i32(refs))
        with torch.cuda.graph(graph):
            step(a, b, torch.cuda.current_stream())
            for k in a:
                a[k].copy_(b[k])
        parents = [-1] * rows
        for i in range(60):
            par.copy_(i32(parents))
            graph.replay()
            torch.cuda.synchronize()
            tables, lens, refs, pairs, st = P.fork(parents, tables, lens, [1] * rows, refs, width)
            assert (a["t"].tolist(), a["n"].tolist(), a["r"].tolist()) == (tables, lens, refs)
            assert [tuple(c) for c in copies.tolist()] == pairs and tuple(status.tolist()) == st
            parents = [rng.randrange(rows) for _ in range(rows)]


# ---- the ends of the ranges -----------------------------------------------------------------------------------------

def test_as_many_rows_and_pages_as_there_may_be():
    """8192 rows continued and moved in a pool of 2^22 pages, by numpy's account of it."""
    rng = np.random.default_rng(31)
    count, n, width = 1 << 22, 8192, 5
    ids = rng.permutation(count)[:n * 4].astype(np.int32)
    lens = rng.integers(1, 65, n).astype(np.int32)
    held = -(-lens // PAGE)
    tables = np.full((n, width), -1, np.int32)
    at = np.concatenate([[0], np.cumsum(held)])
    refs = np.zeros(count, np.int32)
    for r in range(n):
        tables[r, :held[r]] = ids[at[r]:at[r + 1]]
    refs[ids[:at[-1]]] = 1
    parents = np.arange(n)[::-1].copy()     # every row goes on once: nothing is copied or released
    with Pages(count, n, width) as pages:
        got, got_lens, got_refs, copies, status = pages.fork(parents.tolist(), tables.tolist(), lens.tolist(), 16, refs.tolist())
        fresh = np.nonzero(refs == 0)[0][:n]
        want = tables[parents].copy()
        want[np.arange(n), held[parents]] = fresh
        assert np.array_equal(np.array(got), want) and np.array_equal(got_lens, lens[parents] + 16)
        assert all(c == (-1, -1) for c in copies) and status == (0, 0, n, count - int((refs > 0).sum()))
        refs[fresh] = 1
        assert np.array_equal(got_refs, refs)
        # one parent for all: its pages are named 8192 times, and all of the others are free again
        got, got_lens, got_refs, copies, status = pages.fork([7] * n, tables.tolist(), lens.tolist(), 0, (refs * (tables_refs(tables, count) > 0)).tolist())
        full, rest = int(lens[7]) // PAGE, int(lens[7]) % PAGE
        named = np.zeros(count, np.int64)
        np.add.at(named, np.array(got)[np.array(got) >= 0], 1)
        assert np.array_equal(named, got_refs) and (np.array(got)[:, :full] == tables[7, :full]).all()
        assert sum(c[0] >= 0 for c in copies) == (n - 1 if rest else 0)


def tables_refs(tables, count):
    refs = np.zeros(count, np.int64)
    np.add.at(refs, tables[tables >= 0], 1)
    return refs
