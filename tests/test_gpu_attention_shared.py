"""Attention of rows that share prefixes, alone (tdp_stage_attend) and in a decode step (tdp_stage_decode_shared).

The tolerance of an output o = sum p v: a probability is rounded to bf16 (2^-8 of itself at most), so the sum is off by 2^-8 of sum p |v|,
and the output by another 2^-8 of itself.  Scores are fp32 sums of 128 products at most: off by 128 * 2^-24 of sum |q k| / sqrt(dh), below
2^-12 for the inputs here (sum |q k| < 300), which changes a probability by that and the output by twice it: 2^-11 of sum p |v|."""
import numpy as np
import pytest
import torch

from harness import workload as W
from oracle import attend_oracle as A
from paper_2506_10470_amd import tdp
from stage_helpers import TOL, Stage, i32, row_rel_err

pytestmark = pytest.mark.gpu
PAGE = 16
HEADS = {"4/4x64": (4, 4, 64), "8/2x64": (8, 2, 64), "16/1x64": (16, 1, 64), "6/3x128": (6, 3, 128), "16/2x128": (16, 2, 128), "10/2x128": (10, 2, 128),
         "3/3x128": (3, 3, 128), "32/2x128": (32, 2, 128), "14/2x64": (14, 2, 64)}


class Cache:
    """A stage of one layer whose pools hold NaN but for the tokens of the rows: groups of (prefix, [tokens behind it of every row])."""

    def __init__(self, heads, groups, seed=0, kv_scales=None, width=None, max_batch=None, page_share=None):
        hq, hkv, dh = heads
        rng = np.random.default_rng(seed)
        self.heads, self.lens, self.starts, rows = heads, [], [0], []
        lens = [[p + s for s in suffixes] for p, suffixes in groups]
        held = [[-(-n // PAGE) for n in g] for g in lens]
        total = sum(p // PAGE + sum(h - p // PAGE for h in hs) for (p, _), hs in zip(groups, held))
        self.count = total + 5
        ids = rng.permutation(self.count).tolist()
        self.width = width or max([1] + [h for hs in held for h in hs])
        for (p, _), ns, hs in zip(groups, lens, held):
            common = [ids.pop() for _ in range(p // PAGE)]
            rows += [(common + [ids.pop() for _ in range(h - len(common))], n) for h, n in zip(hs, ns)]
            self.starts.append(len(rows))
        self.batch = len(rows)
        self.lens = [n for _, n in rows]
        # entries behind a row's pages are ids that must not be looked up
        self.tables = np.full((self.batch, self.width), -7, np.int32)
        for b, (pages, _) in enumerate(rows):
            self.tables[b, :len(pages)] = pages
        self.scales = kv_scales
        shape = W.StageShape("attend", 1, 64, hq, hkv, dh, 64)
        self.stage = Stage(tdp, shape, self.count, max_batch or max(1, self.batch), 0, 0, self.width, load_weights=False, kv_scales=kv_scales)
        self.stage.poison()
        g = torch.Generator().manual_seed(seed)
        filled = np.zeros(self.count, int)          # slots in use of every page
        for pages, n in rows:
            for j, p in enumerate(pages):
                filled[p] = max(filled[p], min(PAGE, n - j * PAGE))
        k = torch.randn((self.count, hkv, PAGE, dh), generator=g)
        v = torch.randn((self.count, hkv, PAGE, dh), generator=g)
        if kv_scales:
            k, v = ((t / s).clamp(-448, 448).to(torch.float8_e4m3fn) for t, s in ((k, kv_scales[0]), (v, kv_scales[1])))
        else:
            k, v = k.bfloat16(), v.bfloat16()
        self.k, self.v = (t.double().numpy() * s for t, s in zip((k, v), kv_scales or (1.0, 1.0)))
        used = torch.arange(PAGE)[None] < torch.from_numpy(filled)[:, None]
        piece = 64 if kv_scales else 32
        raw = (lambda t: t.view(torch.uint8)) if kv_scales else (lambda t: t)
        pk, pv = self.stage.raw_pools(0)
        pk = pk.view(self.count, hkv, dh // piece, PAGE, piece)
        pv = pv.view(self.count, hkv, dh, PAGE)
        mask = used.cuda()
        kk = raw(k).cuda().view(self.count, hkv, PAGE, dh // piece, piece).permute(0, 1, 3, 2, 4)
        pk.copy_(torch.where(mask[:, None, None, :, None], kk, pk))
        pv.copy_(torch.where(mask[:, None, None, :], raw(v).cuda().permute(0, 1, 3, 2), pv))
        self.q = (torch.randn((self.batch, hq, dh), generator=g) * 1.5).bfloat16()

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.stage.close()

    def attend(self, starts=None, lens=None, stream=None):
        """With the cache's own groups, or others (a list of starts; [] for none)."""
        starts = self.starts if starts is None else starts
        q, out = self.q.cuda(), torch.full(self.q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
        lens, tables, st = i32(self.lens if lens is None else lens), i32(self.tables), i32(starts) if starts else None
        torch.cuda.synchronize()
        tdp.tdp_stage_attend(self.stage.h, 0, q, lens, tables, self.batch, st, max(0, len(starts) - 1), out, stream)
        torch.cuda.synchronize()
        return out

    def check(self, out, lens=None):
        got, q = out.double().cpu().numpy(), self.q.double().numpy()
        for b, n in enumerate(self.lens if lens is None else lens):
            n = min(max(n, 0), PAGE * self.width)
            pages = self.tables[b, :-(-n // PAGE)]
            k, v = (t[pages].transpose(0, 2, 1, 3).reshape(-1, t.shape[1], t.shape[3])[:n] for t in (self.k, self.v))
            o, spread = A.attend(q[b], k, v)
            assert np.isfinite(got[b]).all(), b
            off = np.abs(got[b] - o) - ((2.0 ** -8 + 2.0 ** -11) * spread + 2.0 ** -8 * np.abs(o))
            assert (off <= 0).all(), (b, n, off.max())


MIXED = [(100, [1, 5, 28, 60]), (0, [3]), (64, [16, 1]), (500, [40, 1, 300]), (15, [1, 200, 8]), (33, [15, 15, 16, 17, 31])]


@pytest.mark.parametrize("kv_scales", [None, (0.02, 0.015)])
@pytest.mark.parametrize("heads", HEADS)
def test_groups_of_many_kinds(heads, kv_scales):
    with Cache(HEADS[heads], MIXED, 1, kv_scales) as c:
        out = c.attend()
        c.check(out)
        assert torch.equal(out, c.attend())                 # the same bits again
        c.check(c.attend([]))                               # every row for itself
        c.check(c.attend([0, c.batch]))                     # one group that shares nothing
        c.check(c.attend(list(range(c.batch + 1))))         # groups of one
        c.check(c.attend([0, 0, 4, 4, 7, 10, 13, c.batch, c.batch]))        # empty groups, and borders elsewhere


@pytest.mark.parametrize("kv_scales", [None, (0.02, 0.015)])
@pytest.mark.parametrize("heads", ["4/4x64", "8/2x64", "3/3x128", "16/2x128"])
@pytest.mark.parametrize("rows", [2, 5, 9, 33])
def test_prefixes_of_every_length_around_a_block(heads, rows, kv_scales):
    """Tiles of 16, 64 and 128 columns, prefixes that end in every page of a block."""
    for pages in (1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 32, 33, 49):
        with Cache(HEADS[heads], [(pages * PAGE + pages % 3, [1 + 3 * i % 20 for i in range(rows)])], pages, kv_scales) as c:
            c.check(c.attend())


@pytest.mark.parametrize("heads", ["4/4x64", "16/2x128"])
def test_long_prefixes_in_many_spans(heads):
    for prefix, rows in ((5000, 3), (9000, 20), (4103, 70)):
        with Cache(HEADS[heads], [(prefix, [1 + 7 * i % 50 for i in range(rows)]), (700, [3, 4]), (0, [2])], prefix) as c:
            c.check(c.attend())


def test_a_large_group_of_many_tiles():
    with Cache(HEADS["16/2x128"], [(1100, [1 + 11 * i % 90 for i in range(200)])], 3) as c:
        c.check(c.attend())
    with Cache(HEADS["10/2x128"], [(300, [1 + 11 * i % 40 for i in range(77)]), (320, [1 + i for i in range(51)])], 4) as c:
        c.check(c.attend())


@pytest.mark.parametrize("span", [256, 512, 4096])
@pytest.mark.parametrize("heads", ["8/2x64", "3/3x128"])
def test_rows_of_several_spans_behind_a_prefix(heads, span):
    with Cache(HEADS[heads], [(640, [1, 256, 257, 900, 2000]), (90, [700, 3]), (256, [255, 600]), (250, [256, 6])], 5) as c:
        tdp.tdp_stage_set_decode_span(c.stage.h, span)
        c.check(c.attend())
        c.check(c.attend([]))
        c.check(c.attend())


@pytest.mark.parametrize("kv_scales", [None, (0.02, 0.015)])
@pytest.mark.parametrize("heads", ["8/2x64", "6/3x128"])
def test_partials_that_the_waves_share_out(heads, kv_scales):
    """Rows of up to forty spans, behind prefixes of none, of few and of many; the same bits again."""
    for groups in ([(0, [1800, 2100, 2400, 10000])], [(600, [1, 1500, 1800, 5000, 300])], [(9000, [1, 20, 300, 700])], [(2048, [1, 256, 257, 16])]):
        with Cache(HEADS[heads], groups, 17, kv_scales) as c:
            tdp.tdp_stage_set_decode_span(c.stage.h, 256)
            out = c.attend()
            c.check(out)
            assert all(torch.equal(out, c.attend()) for _ in range(5))


def test_rows_that_fill_their_tables():
    """Spans of the prefix and of the rows together are no more than a row has slots for."""
    for prefix, width in ((16, 16), (16, 33), (256, 32), (272, 33), (1008, 64), (496, 48)):
        with Cache(HEADS["8/2x64"], [(prefix, [width * PAGE - prefix, 1, width * PAGE - prefix])], 6, width=width) as c:
            tdp.tdp_stage_set_decode_span(c.stage.h, 256)
            c.check(c.attend())


def test_rows_without_tokens():
    with Cache(HEADS["8/2x64"], [(100, [1, 5, 28]), (64, [16, 1])], 7) as c:
        for lens in ([0, 105, 128, 80, 65], [101, 0, 0, 0, 0], [0] * 5, [101, -3, 128, 80, 0], [1, 16, 17, 64, 65]):
            for starts in (None, [], [0, 5]):
                out = c.attend(starts, lens)
                c.check(out, lens)
                for b, n in enumerate(lens):
                    assert n > 0 or not out[b].any()
        # what the table of such a row holds is not looked at
        c.tables[0] = c.tables[2] = -7
        lens = [0, 105, 0, 80, 65]
        c.check(c.attend(None, lens), lens)
        c.tables[3] = -7
        lens = [0, 105, 0, 0, 65]
        for starts in (None, [], [0, 5], [0, 1, 5]):
            c.check(c.attend(starts, lens), lens)


def test_identical_tables_share_all_but_the_last_page():
    """Rows that name the same pages throughout (a prompt forked before anything was written): also where a page ends."""
    for n in (1, 16, 17, 64, 100, 300):
        with Cache(HEADS["8/2x64"], [(n // PAGE * PAGE, [n % PAGE or 1])], 8) as c:
            tables, q = i32(np.repeat(c.tables, 6, 0)), c.q.cuda().repeat(6, 1, 1)
            stage = c.stage
            with Stage(tdp, stage.shape, c.count, 6, 0, 0, c.width, load_weights=False) as st:
                for a, b in zip(st.raw_pools(0), stage.raw_pools(0)):
                    a.copy_(b)
                out = torch.empty_like(q)
                tdp.tdp_stage_attend(st.h, 0, q, i32(c.lens * 6), tables, 6, i32([0, 6]), 1, out)
                torch.cuda.synchronize()
                for b in range(6):
                    c.check(out[b:b + 1])


def repeated(c, times, starts_of, span=0):
    """The rows of a cache several times over, with the same queries: {number of groups: output}, for each list of starts."""
    batch, (hq, hkv, dh) = c.batch * times, c.heads
    with Stage(tdp, c.stage.shape, c.count, batch, 0, 0, c.width, load_weights=False) as st:
        for a, b in zip(st.raw_pools(0), c.stage.raw_pools(0)):
            a.copy_(b)
        if span:
            tdp.tdp_stage_set_decode_span(st.h, span)
        q, lens, tables = c.q.cuda().repeat(times, 1, 1), i32(c.lens).repeat(times), i32(c.tables).repeat(times, 1)
        for starts in starts_of:
            out = torch.full_like(q, float("nan"))
            tdp.tdp_stage_attend(st.h, 0, q, lens, tables, batch, i32(starts) if starts else None, max(0, len(starts) - 1), out)
            torch.cuda.synchronize()
            yield out.view(times, c.batch, hq, dh)


@pytest.mark.parametrize("span", [0, 256])
@pytest.mark.parametrize("heads,times", [("4/4x64", 420), ("6/3x128", 260), ("16/1x64", 1100)])
def test_more_rows_and_groups_than_one_workgroup_holds(heads, times, span):
    """Over 1024 rows, and over 1024 groups, some of whose rows have several spans."""
    groups = [(272, [1, 30]), (0, [3]), (600, [1300, 16])]
    with Cache(HEADS[heads], groups, 13) as c:
        n = c.batch * times
        every = [5 * t + s for t in range(times) for s in (0, 2, 3)] + [n]
        assert n > 1024 and (len(every) > 1025) == (times > 341)
        for out in repeated(c, times, (every, [], list(range(n + 1)), [0, 2, 2, 3, 5]), span):
            c.check(out[0])
            c.check(out[-1])
            assert (out[1:-1] == out[1:2]).all()
            c.check(out[1])


def test_one_group_of_more_rows_than_the_comparing_workgroups_hold():
    with Cache((2, 1, 64), [(64, [1, 9, 17, 33, 2])], 14) as c:
        for out in repeated(c, 3400, ([0, 5 * 3400], [0, 3, 5 * 3400 - 2, 5 * 3400])):
            c.check(out[0])
            c.check(out[-1])
            assert (out[1:-1] == out[1:2]).all()
            c.check(out[1])


def test_a_span_of_more_pages_than_a_wave_holds_at_once():
    """Thirteen groups behind 262 to 300 pages, 64 heads: a span each."""
    for pages in (262, 300):
        with Cache((64, 64, 64), [(pages * PAGE, [5, 20])], 15) as c:
            for out in repeated(c, 13, ([2 * g for g in range(14)],)):
                c.check(out[0])
                assert (out == out[:1]).all()


@pytest.mark.parametrize("kv_scales", [None, (0.02, 0.015)])
@pytest.mark.parametrize("rows", [2, 6, 20])
def test_pages_behind_more_elements_than_32_bits_count(rows, kv_scales):
    """The same rows from the first pages of a pool and from the last ones of a pool of over 2^32 elements, where copies have brought them."""
    heads = (64, 8, 128)
    with Cache(heads, [(200, [1 + 7 * i for i in range(rows)]), (0, [40])], 16, kv_scales) as c:
        want, count = c.attend(), (1 << 32) // (8 * 16 * 128) + 500
        with Stage(tdp, c.stage.shape, count, c.batch, 0, 0, c.width, load_weights=False, kv_scales=kv_scales) as st:
            for a, b in zip(st.raw_pools(0), c.stage.raw_pools(0)):
                a.view(-1)[:b.numel()].copy_(b.view(-1))
            moves = [[p, count - 1 - p] for p in range(c.count)]
            tdp.tdp_stage_kv_copy_pages(st.h, i32(moves), len(moves))
            q, out = c.q.cuda(), torch.empty_like(want)
            tables = i32(np.where(c.tables >= 0, count - 1 - c.tables, -7))
            tdp.tdp_stage_attend(st.h, 0, q, i32(c.lens), tables, c.batch, i32(c.starts), len(c.starts) - 1, out)
            torch.cuda.synchronize()
            c.check(want)
            assert torch.equal(out, want)


def test_infinite_and_missing_numbers_stay_where_they_are():
    """A NaN key or an infinite value in one row's own pages, or in one group's prefix, is nobody else's."""
    with Cache(HEADS["8/2x64"], [(100, [1, 5, 28]), (64, [16, 1]), (80, [3, 3])], 9) as c:
        k, v = c.stage.raw_pools(0)
        k = k.view(c.count, -1)
        v = v.view(c.count, 2, 64, PAGE)
        k[int(c.tables[1, 6])] = float("nan")           # of row 1 alone
        v[int(c.tables[3, 0]), :, :, 2] = float("inf")  # of the second group's prefix
        torch.cuda.synchronize()
        out = c.attend()
        assert torch.isnan(out[1]).all() and not torch.isfinite(out[3:5]).any()
        clean = [0, 2, 5, 6]
        want, got = c.attend([]), out
        assert torch.isfinite(got[clean]).all()
        keep = c.lens
        got = got.double().cpu()
        for b in clean:
            pages = c.tables[b, :-(-keep[b] // PAGE)]
            kk, vv = (t[pages].transpose(0, 2, 1, 3).reshape(-1, 2, 64)[:keep[b]] for t in (c.k, c.v))
            o, spread = A.attend(c.q[b].double().numpy(), kk, vv)
            assert (np.abs(got[b].numpy() - o) <= (2.0 ** -8 + 2.0 ** -11) * spread + 2.0 ** -8 * np.abs(o)).all()
        assert torch.isnan(want[1]).all()


def test_pages_are_only_read_and_rows_behind_the_batch_left_alone():
    with Cache(HEADS["16/2x128"], MIXED, 10, max_batch=40) as c:
        before = [t.view(torch.int16).clone() for t in c.stage.raw_pools(0)]
        q = torch.zeros((40, 16, 128), dtype=torch.bfloat16, device="cuda")
        q[:c.batch] = c.q.cuda()
        out = torch.full_like(q, 7.0)
        tdp.tdp_stage_attend(c.stage.h, 0, q, i32(c.lens), i32(c.tables), c.batch, i32(c.starts), len(c.starts) - 1, out)
        torch.cuda.synchronize()
        c.check(out[:c.batch])
        assert (out[c.batch:] == 7.0).all()
        assert all(torch.equal(a, b.view(torch.int16)) for a, b in zip(before, c.stage.raw_pools(0)))


def test_refusals():
    with Cache(HEADS["8/2x64"], [(32, [1, 5])], 11) as c:
        q, n, t, s = c.q.cuda(), i32(c.lens), i32(c.tables), i32(c.starts)
        out = torch.empty_like(q)
        ok = dict(layer=0, q=q, n=n, t=t, b=2, s=s, g=1, out=out)
        for bad in [dict(layer=1), dict(layer=-1), dict(q=None), dict(n=None), dict(t=None), dict(out=None), dict(b=3), dict(b=-1), dict(g=-1), dict(g=3),
                    dict(s=None), dict(q=q.data_ptr() + 8), dict(out=out.data_ptr() + 4)]:
            a = {**ok, **bad}
            with pytest.raises(tdp.TdpError) as e:
                tdp.tdp_stage_attend(c.stage.h, a["layer"], a["q"], a["n"], a["t"], a["b"], a["s"], a["g"], a["out"])
            assert e.value.code == tdp.EINVAL, bad
        for bad in [dict(q=None), dict(n=None), dict(t=None), dict(out=None), dict(b=3), dict(b=-1), dict(g=-1), dict(g=3), dict(s=None)]:
            a = {**ok, **bad}
            with pytest.raises(tdp.TdpError) as e:
                tdp.tdp_stage_decode_shared(c.stage.h, a["q"], a["n"], a["t"], a["b"], a["s"], a["g"], a["out"])
            assert e.value.code == tdp.EINVAL, bad
        tdp.tdp_stage_attend(c.stage.h, 0, None, None, None, 0, None, 0, None)
        tdp.tdp_stage_decode_shared(c.stage.h, None, None, None, 0, None, 0, None)


def test_replayed_with_other_lengths_and_tables():
    with Cache(HEADS["16/2x128"], MIXED, 12) as c:
        q, n, t, s = c.q.cuda(), i32(c.lens), i32(c.tables), i32(c.starts)
        out = torch.empty_like(q)

        def call(stream):
            tdp.tdp_stage_attend(c.stage.h, 0, q, n, t, c.batch, s, len(c.starts) - 1, out, stream)
        call(None)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(torch.cuda.current_stream())
        for i in range(4):
            lens = [max(0, x - 9 * i) for x in c.lens]
            n.copy_(i32(lens))
            out.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            c.check(out, lens)
            want = c.attend(lens=lens)          # eager between the replays
            assert torch.equal(want, out)


# ---- a decode step --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("shape,kv_scales", [("tiny", None), ("tiny_gqa", None), ("tiny_gqa", (0.05, 0.04)), ("tiny_h128", None), ("tiny_mqa", None),
                                             ("tiny_bias", (0.05, 0.04))])
@pytest.mark.parametrize("micro", [0, 2])
def test_a_decode_step_with_groups_is_the_decode_step(shape, kv_scales, micro):
    """Hidden states within the tolerance that the stage's own tests have, and the same keys and values appended."""
    sh = W.SHAPES[shape]
    groups = [(96, [4, 20, 4, 9]), (0, [30]), (340, [1, 33, 16])]
    hidden = W.hidden_states(sh, 8, 77, device="cuda")
    results = []
    for shared in (False, True):
        rng = np.random.default_rng(3)
        count, width = 80, 32
        ids = rng.permutation(count).tolist()
        tables, lens, starts = np.zeros((8, width), np.int32), [], [0]
        b = 0
        for prefix, own in groups:
            common = [ids.pop() for _ in range(prefix // PAGE)]
            for n in own:
                row = common + [ids.pop() for _ in range((prefix + n) // PAGE + 1 - len(common))]
                tables[b, :len(row)] = row
                lens.append(prefix + n)
                b += 1
            starts.append(b)
        with Stage(tdp, sh, count, 8, 0, 0, width, kv_scales=kv_scales, decode_micro_batches=micro) as st:
            g = torch.Generator(device="cuda").manual_seed(5)
            for l in range(sh.n_layers):
                for t in st.raw_pools(l):
                    x = torch.randn(t.shape, generator=g, device="cuda")
                    t.copy_(x.bfloat16() if kv_scales is None else (x / 0.05).to(torch.float8_e4m3fn).view(torch.uint8))
            out = torch.empty_like(hidden)
            args = (st.h, hidden, i32(lens), i32(tables), 8)
            tdp.tdp_stage_check_decode(st.h, i32(lens), i32(tables), 8)
            if shared:
                tdp.tdp_stage_decode_shared(*args, i32(starts), len(groups), out)
            else:
                tdp.tdp_stage_decode(*args, out)
            torch.cuda.synchronize()
            results.append((out.double().cpu().numpy(), [t.view(torch.uint8).clone() for t in st.raw_pools(0)]))
    (want, pools), (got, pools2) = results
    assert row_rel_err(got, want) <= TOL
    assert all(torch.equal(a, b) for a, b in zip(pools, pools2))


def test_a_captured_decode_step_with_groups_follows_its_tables():
    """Replays with other lengths and tables, eager steps between them, each against the step without groups."""
    sh = W.SHAPES["tiny_gqa"]
    rng, count, width, rows = np.random.default_rng(4), 90, 24, 6
    hidden = W.hidden_states(sh, rows, 78, device="cuda")
    starts = i32([0, 4, 6])

    def batch(turn):
        ids = rng.permutation(count).tolist()
        tables, lens = np.zeros((rows, width), np.int32), []
        for b, (group, own) in enumerate(zip((0, 0, 0, 0, 1, 1), (4, 20, 1, 9, 30, 2))):
            if b in (0, 4):
                common = [ids.pop() for _ in range((2 + turn) * (group + 1))]
            n = len(common) * PAGE + own
            row = common + [ids.pop() for _ in range(n // PAGE + 1 - len(common))]
            tables[b, :len(row)] = row
            lens.append(n)
        return i32(lens), i32(tables)

    with Stage(tdp, sh, count, rows, 0, 0, width) as st, Stage(tdp, sh, count, rows, 0, 0, width) as other:
        g = torch.Generator(device="cuda").manual_seed(6)
        for l in range(sh.n_layers):
            for a, b in zip(st.raw_pools(l), other.raw_pools(l)):
                a.copy_(torch.randn(a.shape, generator=g, device="cuda").bfloat16())
                b.copy_(a)
        lens, tables = batch(0)
        out, want = torch.empty_like(hidden), torch.empty_like(hidden)

        def step(stream=None):
            tdp.tdp_stage_decode_shared(st.h, hidden, lens, tables, rows, starts, 2, out, stream)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(torch.cuda.current_stream())
        for turn in range(4):
            for old, new in zip((lens, tables), batch(turn)):
                old.copy_(new)
            for l in range(sh.n_layers):
                for a, b in zip(st.raw_pools(l), other.raw_pools(l)):
                    b.copy_(a)
            out.fill_(float("nan"))
            graph.replay()
            tdp.tdp_stage_decode(other.h, hidden, lens, tables, rows, want)
            torch.cuda.synchronize()
            assert row_rel_err(out.double().cpu().numpy(), want.double().cpu().numpy()) <= TOL
            replayed = out.clone()
            step()
            torch.cuda.synchronize()
            assert torch.equal(replayed, out)
