"""Beam selection on the GPU against the oracle in 64 bits.

A row's sum of exponentials is of terms that are off by 2^-23 (the instruction) and 2^-24 (the argument's rounding, |d| 2^-24 of a term that
is at most e^d: below 2^-24 in all), summed in fp32 in chains of 64 at most: in the worst case (64 + 3) 2^-24 of the sum, and so of a
score, apart from the score's own rounding to fp32, 2^-24 of itself."""
import numpy as np
import pytest
import torch

from oracle import beams_oracle as B
from paper_2506_10470_amd import tdp

pytestmark = pytest.mark.gpu
INF = float("inf")
TOL = 67 * 2.0 ** -24


class Beams:
    def __init__(self, rows=64, out=32):
        self.h = tdp.tdp_beams_create(tdp.BeamsConfig(rows, out))

    def __enter__(self):
        return self

    def __exit__(self, *a):
        tdp.tdp_beams_destroy(self.h)

    def select(self, logits, scores, beams, n_out, finished=None, end=-1, n=None, stream=None, flags=True):
        groups = len(scores) // beams
        parent, token, done = (torch.full((max(1, groups), n_out), -9, dtype=torch.int32, device="cuda") for _ in range(3))
        score = torch.full((max(1, groups), n_out), 9.0, device="cuda")
        fin = None if finished is None else torch.as_tensor(finished, dtype=torch.int32, device="cuda")
        tdp.tdp_beams_select(self.h, logits, tdp.BF16 if logits.dtype == torch.bfloat16 else tdp.F32, groups, beams, n or logits.shape[1],
                             logits.stride(0), torch.as_tensor(scores, dtype=torch.float32, device="cuda"), fin, end, n_out, parent, token, score,
                             done if flags else None, stream)
        torch.cuda.synchronize()
        return [x.cpu().numpy() for x in (parent, token, score, done)]


def check(got, logits, scores, beams, n_out, finished=None, end=-1):
    """Every place holds a candidate that is as good as the oracle's within the tolerance, and the oracle's own where no other is that close."""
    parent, token, score, done = got
    z = logits.double().cpu().numpy()
    scores = np.asarray(scores, np.float32).astype(np.float64)
    want_parent, want_token, want, want_done = B.select(z, scores, beams, n_out, finished, end)
    c = B.candidates(z, scores, finished, end)
    real = want_parent >= 0
    assert np.array_equal(parent >= 0, real) and np.array_equal(token >= 0, real)
    assert (score[~real] == -INF).all() and (done[~real] == 0).all()
    value = np.where(real, c[parent, token], -INF)
    exact = np.isposinf(want)
    assert (np.abs(value[real & ~exact] - want[real & ~exact]) <= 2 * TOL).all()
    assert (np.abs(score[real & ~exact] - value[real & ~exact]) <= TOL + 2.0 ** -24 * np.abs(value[real & ~exact])).all()
    groups = parent // beams
    assert all((g[p >= 0] == i).all() for i, (g, p) in enumerate(zip(groups, parent)))
    for p, t in zip(parent, token):
        chosen = [(a, b) for a, b in zip(p, t) if a >= 0]
        assert len(set(chosen)) == len(chosen)
    assert np.array_equal(done, (token == end) & real)
    same = (parent == want_parent) & (token == want_token)
    for g, j in zip(*np.nonzero(~same)):  # a near tie, not an exact one
        assert value[g, j] != want[g, j] or c[parent[g, j]].tolist() != c[want_parent[g, j]].tolist()
    return same


def rows(seed, m, n, dtype=torch.float32, spread=2.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn((m, n), generator=g, device="cuda") * spread
    z[:, :: max(1, n // 7)] += 6.0
    return z.to(dtype), (-torch.randn(m, generator=g, device="cuda").abs() * 3 - 5).tolist()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("groups,beams,n,n_out", [
    (1, 1, 1, 1), (1, 4, 1000, 4), (3, 2, 7, 14), (2, 5, 128256, 10), (3, 32, 50, 32), (1, 32, 33001, 32), (7, 3, 5, 15), (40, 8, 3203, 16), (5, 1, 300001, 1),
    (600, 1, 1500, 2), (9, 7, 32768, 7), (33, 16, 4999, 16), (1, 1, 1000003, 32), (1, 3, 31, 32)])
def test_random_rows(groups, beams, n, n_out, dtype):
    z, scores = rows(groups * 31 + n, groups * beams, n, dtype)
    with Beams(groups * beams, n_out) as b:
        got = b.select(z, scores, beams, n_out)
        same = check(got, z, scores, beams, n_out)
        assert same.mean() >= 0.99
        again = b.select(z, scores, beams, n_out)
        assert all(np.array_equal(x, y) for x, y in zip(got, again))


@pytest.mark.parametrize("dtype,n", [(torch.float32, 300_000), (torch.bfloat16, 600_001)])
def test_rows_that_a_workgroup_reads_in_turns(dtype, n):
    z, scores = rows(3, 64, n, dtype)
    with Beams(64, 4) as b:
        check(b.select(z, scores, 2, 4), z, scores, 2, 4)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_at_any_alignment_and_distance(dtype):
    z, scores = rows(5, 12, 2100, dtype)
    with Beams(12, 8) as b:
        for off in range(9):
            for n in (1, 3, 2003, 2049):
                view = z[:, off:off + n]
                assert view.stride(0) == 2100
                check(b.select(view, scores, 4, min(8, 4 * n), n=n), view, scores, 4, min(8, 4 * n))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [40, 5000, 70001])
def test_equal_candidates_go_by_beam_and_token(dtype, n):
    with Beams(8, 32) as b:
        z = torch.zeros((8, n), dtype=dtype, device="cuda")
        parent, token, score, _ = b.select(z, [0.0] * 8, 4, 32)
        assert parent.tolist() == [[0] * 32, [4] * 32] and token.tolist() == [list(range(32))] * 2
        # beams that are the same row: every token first from the lower beam
        # (with n odd they lie at different alignments: their sums have to be the same bits all the same)
        for seed in range(6):
            g = torch.Generator(device="cuda").manual_seed(seed)
            z[:] = (torch.randperm(n, generator=g, device="cuda") % 64 + torch.rand(n, generator=g, device="cuda")).to(dtype)
            want = B.select(z.double().cpu().numpy(), np.zeros(8), 4, 32)
            got = b.select(z, [0.0] * 8, 4, 32)
            assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
        # coarse logits, the same level in all rows: equal within a row, never across them
        z = torch.randint(-8, 8, (8, n), generator=torch.Generator(device="cuda").manual_seed(7), device="cuda").to(dtype)
        check(b.select(z, [-1.0, -1.25, -1.5, -1.75] * 2, 4, 32), z, [-1.0, -1.25, -1.5, -1.75] * 2, 4, 32)


def test_masks_and_rows_without_a_distribution():
    n = 3001
    z, scores = rows(8, 16, n)
    z[0] = -INF                                   # nothing is left
    z[1] = -INF
    z[1, 77] = -3.0                               # one token
    z[2, ::2] = -INF
    z[3, 5] = float("nan")
    z[4, 6] = INF
    z[5] = torch.finfo(torch.float32).min         # the type's lowest value, everywhere
    z[6, 3:] = torch.finfo(torch.float32).min
    scores[7] = -INF
    scores[8] = float("nan")
    z[12:16] = -INF                               # a whole group
    with Beams(16, 32) as b:
        for n_out in (1, 4, 32):
            check(b.select(z, scores, 4, n_out), z, scores, 4, n_out)
        assert (b.select(z, scores, 4, 32)[0][3] == -1).all()
        got = b.select(z[:4], scores[:4], 4, 3)
        assert 77 in got[1][0].tolist() or got[2][0].min() > scores[1]
        zb = z.bfloat16()
        check(b.select(zb, scores, 4, 32), zb, scores, 4, 32)
        few = torch.full((2, 9000), -INF, device="cuda")
        few[0, 8999], few[1, 0] = 1.0, -4.0
        got = b.select(few, [-1.0, -2.0], 2, 5)
        assert got[0].tolist() == [[0, 1, -1, -1, -1]] and got[1].tolist() == [[8999, 0, -1, -1, -1]]
        assert got[2].tolist() == [[-1.0, -2.0, -INF, -INF, -INF]]


@pytest.mark.parametrize("n", [5, 1000, 40000])
def test_finished_beams(n):
    z, scores = rows(13, 24, n)
    z[1] = float("nan")                            # (no matter: it is finished)
    finished = [1 if i % 5 == 1 or i >= 20 else 0 for i in range(24)]
    with Beams(24, 16) as b:
        for end in (0, n - 1, 2):
            got = b.select(z, scores, 4, 8, finished, end)
            check(got, z, scores, 4, 8, finished, end)
            assert (got[0][5] >= 0).sum() == 4 and (got[1][5][:4] == end).all() and (got[3][5] == [1] * 4 + [0] * 4).all()
            assert np.array_equal(got[2][5][:4], np.sort(np.float32(scores[20:]))[::-1])
        got = b.select(z[2:4], scores[2:4], 2, 4, None, 3)      # the end token is told apart without finished beams
        check(got, z[2:4], scores[2:4], 2, 4, None, 3)
        assert b.select(z[2:4], scores[2:4], 2, 4, None, 3, flags=False)[1].tolist() == got[1].tolist()


def test_large_and_small_numbers():
    z, scores = rows(21, 8, 4000)
    with Beams(8, 8) as b:
        for scale, shift in ((1, 1e6), (1, -1e6), (1e4, 0), (1e-3, 0), (0, 88)):
            x = z * scale + shift
            check(b.select(x, scores, 4, 8), x, scores, 4, 8)
        check(b.select(z, [s * 1e4 for s in scores], 4, 8), z, [s * 1e4 for s in scores], 4, 8)


def test_columns_behind_the_row_are_not_read():
    z, scores = rows(4, 8, 1024)
    z[:, 1000:] = float("nan")
    with Beams(8, 8) as b:
        check(b.select(z, scores, 4, 8, n=1000), z[:, :1000], scores, 4, 8)


def test_refusals_and_nothing_to_do():
    z, s = torch.zeros((8, 16), device="cuda"), torch.zeros(8, device="cuda")
    i, f = torch.zeros(64, dtype=torch.int32, device="cuda"), torch.zeros(64, device="cuda")
    with Beams(8, 8) as b:
        ok = dict(z=z, dtype=0, groups=2, beams=4, n=16, ld=16, s=s, fin=None, end=-1, out=4, p=i, t=i, sc=f)
        for bad in [dict(z=None), dict(z=z.data_ptr() + 2), dict(dtype=2), dict(groups=-1), dict(groups=3), dict(beams=0), dict(beams=33), dict(n=0),
                    dict(n=17), dict(n=(1 << 27) + 1, ld=1 << 28), dict(s=None), dict(end=16), dict(end=-2), dict(fin=i), dict(out=0), dict(out=9),
                    dict(n=1, ld=16, out=5), dict(p=None), dict(t=None), dict(sc=None)]:
            a = {**ok, **bad}
            with pytest.raises(tdp.TdpError) as e:
                tdp.tdp_beams_select(b.h, a["z"], a["dtype"], a["groups"], a["beams"], a["n"], a["ld"], a["s"], a["fin"], a["end"], a["out"], a["p"],
                                     a["t"], a["sc"])
            assert e.value.code == tdp.EINVAL, bad
        tdp.tdp_beams_select(b.h, None, 0, 0, 4, 16, 16, None, None, -1, 4, None, None, None)


def test_replayed_on_another_stream():
    z, scores = rows(17, 16, 20000)
    with Beams(16, 8) as b:
        x, s = z.clone(), torch.tensor(scores, device="cuda")
        parent, token = (torch.empty((4, 8), dtype=torch.int32, device="cuda") for _ in range(2))
        score = torch.empty((4, 8), device="cuda")

        def call(stream):
            tdp.tdp_beams_select(b.h, x, tdp.F32, 4, 4, 20000, 20000, s, None, -1, 8, parent, token, score, None, stream)
        call(None)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(torch.cuda.current_stream())
        for seed in (30, 31, 32, 33):
            z, scores = rows(seed, 16, 20000)
            x.copy_(z)
            s.copy_(torch.tensor(scores, device="cuda"))
            graph.replay()
            torch.cuda.synchronize()
            check([parent.cpu().numpy(), token.cpu().numpy(), score.cpu().numpy(), (token == -1).int().cpu().numpy()], z, scores, 4, 8)


# ---- the ends of the ranges -----------------------------------------------------------------------------------------

def test_as_many_rows_as_there_may_be():
    """2048 groups of 32 beams, each the same as its neighbours."""
    z, s = rows(20, 32, 40)
    with Beams(1 << 16, 32) as b:
        got = b.select(z.repeat(2048, 1), s * 2048, 32, 32)
        for x in got[1:]:
            assert (x == x[0]).all()
        assert (got[0] - 32 * np.arange(2048)[:, None] == got[0][0]).all()
        check([x[:1] for x in got], z, s, 32, 32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_longest_row(dtype):
    """2^27 equal logits but for three: the sum is known."""
    n = 1 << 27
    z = torch.zeros((1, n), dtype=dtype, device="cuda")
    z[0, 5], z[0, n - 1], z[0, n // 2 + 1] = 3.0, 4.0, 3.0
    total = np.log(n - 3 + 2 * np.exp(3.0) + np.exp(4.0))
    with Beams(1, 5) as b:
        parent, token, score, _ = b.select(z, [-1.0], 1, 5)
    assert token.tolist() == [[n - 1, 5, n // 2 + 1, 0, 1]] and (parent == 0).all()
    want = np.array([4.0, 3.0, 3.0, 0.0, 0.0]) - 1.0 - total
    assert (np.abs(score[0] - want) <= TOL + 2.0 ** -24 * np.abs(want)).all()


def test_rows_further_apart_than_32_bits_count():
    z, s = rows(21, 4, 3000, torch.bfloat16)
    far = torch.empty(3 * (1 << 30) + (3 << 4) + 3000, dtype=torch.bfloat16, device="cuda")
    far = far.as_strided((4, 3000), ((1 << 30) + 16, 1))
    far.copy_(z)
    with Beams() as b:
        for x, y in zip(b.select(far, s, 2, 6), b.select(z, s, 2, 6)):
            assert np.array_equal(x, y)


def test_two_objects_on_two_streams_at_once():
    inputs = [rows(22 + i, 32, 40000 + i) for i in range(2)]
    with Beams() as one, Beams() as two:
        want = [b.select(z, s, 4, 8) for b, (z, s) in zip((one, two), inputs)]
        streams = [torch.cuda.Stream() for _ in range(2)]
        scores = [torch.tensor(s, device="cuda") for _, s in inputs]
        outs = [[[torch.empty((8, 8), dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32)] for _ in range(20)] for _ in range(2)]
        torch.cuda.synchronize()
        for turn in range(20):
            for b, (z, _), s, st, out in zip((one, two), inputs, scores, streams, outs):
                tdp.tdp_beams_select(b.h, z, tdp.F32, 8, 4, z.shape[1], z.shape[1], s, None, -1, 8, *out[turn], None, st)
        torch.cuda.synchronize()
        for w, out in zip(want, outs):
            for got in out:
                assert all(np.array_equal(a, t.cpu().numpy()) for a, t in zip(w, got))
