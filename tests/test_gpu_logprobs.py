"""Log-probabilities of given logits (tdp_logprob_rows) and behind the vocabulary projection (tdp_lm_head_logprobs), against
oracle/logprob_oracle.py.  Tokens are exact; tolerances are the oracle's `tolerance`, derived from fp32 roundings there, and two roundings
of the result itself."""
import numpy as np
import pytest
import torch

from harness import workload as W
from oracle import ends_oracle as E
from oracle import int8_oracle as Q
from oracle import logprob_oracle as L
from paper_2506_10470_amd import tdp
from stage_helpers import f64, i32

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def call(logits, dtype, M, n, ld, targets, n_top, stream=None):
    """(logprob, entropy, index, top_logprob) as numpy arrays, from poisoned results"""
    lp = torch.full((M,), 777.0, device="cuda")
    en = torch.full((M,), 777.0, device="cuda")
    ix = torch.full((M, n_top), 777, dtype=torch.int32, device="cuda")
    tl = torch.full((M, n_top), 777.0, device="cuda")
    t = None if targets is None else i32(targets)
    tdp.tdp_logprob_rows(logits, dtype, M, n, ld, t, n_top, lp, en, ix if n_top else None, tl if n_top else None, stream)
    torch.cuda.synchronize()
    return [a.cpu().numpy() for a in (lp, en, ix, tl)]


def near(got, ref, tol):
    """Equal where not finite, else within tol and two roundings of the value"""
    got, ref = np.asarray(got, dtype=np.float64), np.asarray(ref, dtype=np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), (got, ref)
    # (a value beyond fp32's largest, (2 - 2^-23) 2^127, by half a step or more rounds to infinity: -3e38 - 3e38 is no fp32 number)
    ref = np.where(np.abs(ref) >= (2 - 2.0 ** -24) * 2.0 ** 127, np.copysign(np.inf, ref), ref)
    inf = np.isinf(ref)
    assert np.array_equal(got[inf], ref[inf])
    fine = np.isfinite(ref)
    tol = np.broadcast_to(tol, ref.shape)
    off = np.abs(got[fine] - ref[fine]) - (tol[fine] + 2 * U * np.abs(ref[fine]))
    assert (off <= 0).all(), (off.max(), got[fine][off.argmax()], ref[fine][off.argmax()])


def check(got, z, targets, n_top):
    z = np.asarray(z, dtype=np.float64)
    lp, en, ix, tl = L.answer(z, targets, n_top)
    of_log, of_entropy = L.tolerance(z)
    assert np.array_equal(got[2], ix)
    near(got[0], lp, of_log)
    near(got[1], en, of_entropy)
    near(got[3], tl, of_log[:, None])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,n,ld,shift,n_top", [
    (1, 1, 1, 0, 1), (3, 2, 2, 0, 2), (5, 7, 9, 1, 3), (4, 33, 33, 0, 32), (2, 63, 64, 3, 20), (3, 64, 64, 0, 32), (3, 65, 65, 0, 32),
    (7, 255, 257, 5, 5), (2, 1000, 1000, 0, 0), (9, 1003, 1010, 2, 32), (2, 4097, 4097, 0, 1), (3, 8191, 8191, 7, 20),
    (2, 16385, 16385, 0, 5), (3, 32000, 32000, 0, 20), (2, 32003, 32003, 1, 32), (2, 151936, 151936, 0, 32), (1, 300001, 300001, 1, 20)])
def test_sizes_and_alignments(M, n, ld, shift, n_top, dtype):
    """Rows that begin and end anywhere in a 16-byte vector, between numbers that must not count (the padding is larger than any logit)."""
    g = torch.Generator().manual_seed(M * 1000 + n)
    flat = torch.full((shift + M * ld + 8,), 1000.0)
    z = torch.randn(M, n, generator=g) * 3
    z = z.to(dtype)
    rows = flat[shift:shift + M * ld].view(M, ld)
    rows[:, :n] = z.float()
    dev = flat.to(dtype).cuda()[shift:]
    targets = torch.randint(0, n, (M,), generator=g).numpy()
    kind = tdp.F32 if dtype == torch.float32 else tdp.BF16
    check(call(dev, kind, M, n, ld, targets, n_top), f64(z), targets, n_top)
    check(call(dev, kind, M, n, ld, None, n_top), f64(z), None, n_top)


def special_rows(n, seed):
    """Rows where masks and ties decide; every one is documented by its name"""
    rng = np.random.default_rng(seed)
    base = (rng.standard_normal(n) * 2).astype(np.float32)
    inf, low = np.float32(np.inf), np.finfo(np.float32).min
    rows = {}
    rows["all equal"] = np.zeros(n, np.float32)
    rows["both zeros"] = np.where(np.arange(n) % 3 == 0, np.float32(-0.0), np.float32(0.0))
    rows["nothing left"] = np.full(n, -inf, np.float32)
    r = np.full(n, -inf, np.float32); r[n - 1] = -3.0
    rows["one token, the last"] = r
    r = np.full(n, -inf, np.float32); r[rng.choice(n, min(n, 3), replace=False)] = [1.0, 2.0, 2.0][:min(n, 3)]
    rows["fewer tokens than asked for"] = r
    r = np.full(n, low, np.float32); r[n // 2] = 1.0
    rows["masked with the lowest value"] = r
    rows["nothing but the lowest value"] = np.full(n, low, np.float32)
    r = np.full(n, low, np.float32); r[::2] = -inf
    rows["lowest values and minus infinity"] = r
    r = base.copy(); r[n // 3] = np.nan
    rows["a NaN"] = r
    rows["nothing but NaN"] = np.full(n, np.nan, np.float32)
    r = np.full(n, np.nan, np.float32); r[n // 2] = -inf
    rows["NaN and minus infinity"] = r
    r = base.copy(); r[n // 4] = inf
    rows["plus infinity"] = r
    rows["sorted"] = np.sort(base)[::-1].copy()
    rows["few values"] = rng.integers(-2, 3, n).astype(np.float32)
    rows["large"] = base * np.float32(1e4)
    rows["huge"] = np.where(rng.random(n) < 0.5, np.float32(3e38), np.float32(-3e38))
    r = np.full(n, -30.0, np.float32); r[:max(1, n // 7)] = base[:max(1, n // 7)]
    rows["mass in front"] = r
    # the largest logits all in what a few threads read: every vector whose number is 0 or 1 modulo 64, ..., modulo 1024
    for step in (64, 256, 1024):
        v = (np.arange(n) // 4) % step
        rows["strided %d" % step] = np.where(v < 2, 5 + np.abs(base), base).astype(np.float32)
    return rows


@pytest.mark.parametrize("n", [5, 100, 4100, 32000, 150004])
@pytest.mark.parametrize("n_top", [1, 5, 32])
def test_masks_ties_and_rows_without_a_distribution(n, n_top):
    n_top = min(n, n_top)
    rows = special_rows(n, n)
    z = np.stack(list(rows.values()))
    targets = [(7 * i) % n for i in range(len(z))]
    targets[3], targets[4], targets[5] = -1, n, n + 5
    check(call(torch.from_numpy(z).cuda(), tdp.F32, len(z), n, n, targets, n_top), z, targets, n_top)
    zb = torch.from_numpy(z).to(torch.bfloat16)
    check(call(zb.cuda(), tdp.BF16, len(z), n, n, targets, n_top), f64(zb), targets, n_top)


@pytest.mark.parametrize("n,step,few", [(1 << 20, 1024, 16), ((1 << 20) + 3, 1024, 1), (131072, 1024, 31), (4096, 512, 100)])
@pytest.mark.parametrize("n_top", [2, 20, 32])
def test_large_logits_that_ascend_in_what_a_few_threads_read(n, step, few, n_top):
    """All large logits in every step-th few vectors, larger and larger: no list of those at hand comes near the largest of the row."""
    rng = np.random.default_rng(n + few)
    large = (np.arange(n) // 4) % step < few
    z = -1 - rng.random(n).astype(np.float32)
    z[large] = np.float32(1) + np.arange(large.sum(), dtype=np.float32) * np.float32(2.0 ** -18)  # (exact: below 2^18 of them)
    z = np.stack([z, np.where(large, z, np.float32(-np.inf)), -np.abs(z), np.where(rng.random(n) < 0.001, np.float32(np.nan), z)])
    check(call(torch.from_numpy(z).cuda(), tdp.F32, len(z), n, n, None, n_top), z, None, n_top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,value", [((1 << 22) + 5, -1.0), ((1 << 22) + 5, -1.5), ((1 << 24) + 5, -0.25), ((1 << 24) + 5, -0.5),
                                     ((1 << 24) + 5, -1.0)])
def test_sums_of_many_like_terms(n, value, dtype):
    """Every thread's first logits are the row's largest, all others alike: added one by one to a single fp32 number, each of them would
    be rounded the same way as long as that number has the same exponent, thousands of times.  Maxima rise once: 24 links."""
    top = 8192
    for shift in (0, 3):
        z = torch.full((shift + n,), value, dtype=dtype, device="cuda")
        z[:shift + top] = 0
        lp, en, _, _ = call(z[shift:], tdp.F32 if dtype == torch.float32 else tdp.BF16, 1, n, n, [n - 1], 0)
        e = np.exp(value)
        s = top + (n - top) * e
        of_log, of_entropy = L.tolerance(f64(z[shift:])[None], links=24)
        near(lp, [value - np.log(s)], of_log)
        near(en, [np.log(s) - (n - top) * e * value / s], of_entropy)


def test_a_long_row_that_rises_to_its_end():
    n = (1 << 22) + 3
    z = (np.arange(n) * 2.0 ** -18).astype(np.float32)[None]      # (exact)
    check(call(torch.from_numpy(z).cuda(), tdp.F32, 1, n, n, [n - 9], 2), z, [n - 9], 2)


def test_more_rows_than_a_launch_has_threads_for():
    """70 million rows of four: 2^32 threads and more"""
    M, n = 70_000_000, 4
    z = torch.randn(M, n, device="cuda")
    t = torch.randint(0, n, (M,), device="cuda", dtype=torch.int32)
    lp, ix, tl = torch.empty(M, device="cuda"), torch.empty((M, 1), dtype=torch.int32, device="cuda"), torch.empty((M, 1), device="cuda")
    tdp.tdp_logprob_rows(z, tdp.F32, M, n, n, t, 1, lp, None, ix, tl)
    ref = torch.log_softmax(z, 1)
    assert (lp - ref.gather(1, t.long()[:, None])[:, 0]).abs().max().item() <= 1e-4      # (both in fp32: 400 u of up to 20 each)
    assert torch.equal(ix[:, 0].long(), z.argmax(1))
    assert (tl[:, 0] - ref.max(1).values).abs().max().item() <= 1e-4


def test_results_that_are_not_wanted_are_not_written_and_empty_calls_do_nothing():
    z = torch.randn(4, 50, device="cuda")
    en = torch.full((4,), 7.0, device="cuda")
    tdp.tdp_logprob_rows(z, tdp.F32, 4, 50, 50, None, 0, None, en, None, None)
    ix, tl = torch.full((6, 2), 9, dtype=torch.int32, device="cuda"), torch.full((6, 2), 9.0, device="cuda")
    tdp.tdp_logprob_rows(z, tdp.F32, 4, 50, 50, None, 2, None, None, ix, tl)
    tdp.tdp_logprob_rows(None, tdp.F32, 0, 50, 50, None, 2, None, None, ix, tl)
    torch.cuda.synchronize()
    _, ref, index, top = L.answer(f64(z), None, 2)
    near(en.cpu().numpy(), ref, L.tolerance(f64(z))[1])
    assert np.array_equal(ix.cpu().numpy()[:4], index) and (ix[4:] == 9).all() and (tl[4:] == 9).all()


# ---- behind the vocabulary projection ------------------------------------------------------------------------------------------

class Head:
    def __init__(self, vocab, d, max_tokens, int8, seed=3):
        g = torch.Generator(device="cuda").manual_seed(seed + vocab + d)
        self.vocab, self.d, self.int8 = vocab, d, int8
        self.weights = (torch.randn(d, vocab, generator=g, device="cuda") * 2 / d ** 0.5).to(torch.bfloat16)
        self.gain = 1 + 0.1 * torch.randn(d, generator=g, device="cuda")
        self.h = tdp.tdp_ends_create(tdp.EndsConfig(vocab, d, 1e-5, max_tokens))
        tdp.tdp_ends_set_weight(self.h, tdp.E_FINAL_NORM, self.gain, tdp.F32, tdp.DEVICE, d, 1)
        self.set(int8)

    def set(self, int8):
        tdp.tdp_ends_set_weight(self.h, tdp.E_LM_HEAD_I8 if int8 else tdp.E_LM_HEAD, self.weights, tdp.BF16, tdp.DEVICE, self.d, self.vocab)

    def rows(self, n, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        return torch.randn(n, self.d, generator=g, device="cuda").to(torch.bfloat16)

    def logits(self, x, M, idx=None):
        lg = torch.full((M, self.vocab), float("nan"), device="cuda")
        tok = torch.full((M,), -1, dtype=torch.int32, device="cuda")
        tdp.tdp_lm_head(self.h, x, x.shape[0], idx, M, lg, tok)
        return lg, tok

    def logprobs(self, x, M, targets, n_top, want_token=True, idx=None, stream=None):
        lp, en = torch.full((M,), 7.0, device="cuda"), torch.full((M,), 7.0, device="cuda")
        tok = torch.full((M,), -1, dtype=torch.int32, device="cuda")
        ix, tl = torch.full((M, n_top), 7, dtype=torch.int32, device="cuda"), torch.full((M, n_top), 7.0, device="cuda")
        tdp.tdp_lm_head_logprobs(self.h, x, x.shape[0], idx, M, None if targets is None else i32(targets), n_top,
                                 tok if want_token else None, lp, en, ix if n_top else None, tl if n_top else None, stream)
        return lp, en, ix, tl, tok

    def close(self):
        tdp.tdp_ends_destroy(self.h)

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("M,vocab,d", [(1, 260, 64), (3, 4, 64), (5, 1000, 320), (33, 4100, 256), (48, 32000, 1088), (200, 4004, 128),
                                       (257, 32000, 64), (512, 8004, 192), (700, 2052, 256)])
def test_statistics_in_the_projections_epilogue_are_those_of_its_logits(M, vocab, d, int8):
    """With tokens asked for and without (the logits are then not stored), one target per row or the greedy token's; all kinds of tiles,
    split and unsplit, vocabularies that end inside a tile."""
    n_top = min(vocab, 7)
    with Head(vocab, d, M, int8) as head:
        x = head.rows(M, 5)
        lg, tok = head.logits(x, M)
        rng = np.random.default_rng(1)
        targets = rng.integers(0, vocab, M)
        targets[0], targets[-1] = vocab - 1, -1
        z = lg.cpu().numpy()
        for t in (targets, None):
            lp, en, ix, tl, tok2 = head.logprobs(x, M, t, n_top)
            check([a.cpu().numpy() for a in (lp, en, ix, tl)], z, t, n_top)
            assert torch.equal(tok, tok2)
            lp2, en2, *_ = head.logprobs(x, M, t, 0, want_token=False)
            assert torch.equal(lp, lp2) and torch.equal(en, en2)


def plan_of_head(M, vocab, d):
    """How a bf16 vocabulary projection is made, with the workspace that an ends object for M rows has"""
    padded = -(-vocab // 256) * 256
    return tdp.tdp_gemm_plan(M, vocab, d, 0, False, 2 * min((M + 1) // 2 * 2, 512) * padded)


# batches whose bf16 projection is made in tiles of every kind, unsplit; in chunks of K; and split
BY_TILE = [(20, 8004, 64), (50, 32000, 128), (120, 32000, 320), (129, 8004, 64), (129, 16000, 64), (129, 32000, 64), (194, 16000, 64),
           (194, 64000, 64), (324, 16000, 64), (324, 32000, 64), (454, 16000, 64), (454, 32000, 64), (1026, 8004, 64), (250, 32000, 512),
           (33, 4100, 1152), (64, 8004, 2048), (100, 32000, 2048), (128, 2052, 4096), (16, 32000, 4096)]


def test_the_batches_above_cover_the_kinds_of_tiles():
    plans = [plan_of_head(*c) for c in BY_TILE]
    assert {p["tile"] for p in plans if p["splits"] == 1 and not p["chunk_k"]} == {1, 3, 4, 5, 6, 7, 8, 9, 10, 12, 13}
    assert {p["tile"] for p in plans if p["chunk_k"]} >= {11, 13} and any(p["splits"] > 1 for p in plans)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("M,vocab,d", BY_TILE)
def test_statistics_of_every_kind_of_tile(M, vocab, d, int8):
    """Against log-probabilities of the call's own logits in 64 bits, on the GPU.  (Tolerances as the oracle's, for logits whose spread R is
    at most 40, D at most R: (2 R + 2 + 2 R + 72 + 200 + 2 ln n) u < 500 u and, of the entropy, (1 + R)(...) u.)"""
    with Head(vocab, d, M, int8) as head:
        x = head.rows(M, 5)
        lg, _ = head.logits(x, M)
        targets = np.random.default_rng(M).integers(0, vocab, M)
        lp, en, *_ = head.logprobs(x, M, targets, 0, want_token=False)
        z = lg.double()
        assert (z.max() - z.min()).item() <= 40
        ref = torch.log_softmax(z, 1)
        at = torch.from_numpy(targets).cuda()[:, None]
        entropy = -(ref.exp() * ref).sum(1)
        R = 40
        assert ((lp - ref.gather(1, at)[:, 0]).abs() <= (4 * R + 274 + 2 * np.log(vocab)) * U + 2 * U * R).all()
        assert ((en - entropy).abs() <= (1 + R) * (4 * R + 300 + 2 * np.log(vocab)) * U).all()
        # the tokens, where logits are stored, from the same tiles
        lp2, en2, ix, tl, tok = head.logprobs(x, M, targets, 6)
        assert torch.equal(lp, lp2) and torch.equal(en, en2)
        top = lg.sort(stable=True, dim=1, descending=True)
        assert torch.equal(ix.long(), top.indices[:, :6]) and torch.equal(tok.long(), top.indices[:, 0])
        assert ((tl - ref.gather(1, top.indices[:, :6])).abs() <= 600 * U + 2 * U * R).all()


@pytest.mark.parametrize("M", [1, 20, 300])
def test_logits_of_an_8_bit_head_are_the_quantised_products(M):
    """RMSNorm folds into the scale: codes of x * gain (exact), scale times 1 / rms.  The norm's factor and the three roundings of a logit
    are within 8 u (u = 2^-24; the mean of d squares adds log2(d) + 12 links of a chain, halved by the root: 16 u), the sum is exact."""
    vocab, d = 1004, 320
    with Head(vocab, d, M, True) as head:
        x = head.rows(M, 9)
        x[0] = 0
        lg, _ = head.logits(x, M)
        xs = x.float().cpu().numpy()
        xc, xsc = Q.quantise(xs * head.gain.cpu().numpy())
        wc, wsc = Q.quantise(head.weights.float().cpu().numpy().T)
        rms = 1 / np.sqrt((xs.astype(np.float64) ** 2).mean(1) + 1e-5)
        ref = Q.product(xc, xsc.astype(np.float64) * rms, wc, wsc)
        assert (np.abs(lg.cpu().numpy() - ref) <= 24 * U * np.abs(ref)).all()


def test_an_8_bit_head_is_close_to_the_bf16_one_and_can_be_set_back():
    """Each factor of a product is off by at most half a scale, a / 254 of the vector's largest magnitude a.  Summed at random over d terms
    of magnitudes about a quarter of a, with the bf16 rounding of the norm far below: the logits' distance is 1 to 2 % of their norm."""
    M, vocab, d = 64, 4000, 512
    with Head(vocab, d, M, False) as head:
        x = head.rows(M, 1)
        a, _ = head.logits(x, M)
        head.set(True)
        b, _ = head.logits(x, M)
        head.set(False)
        c, _ = head.logits(x, M)
        assert torch.equal(a, c)
        assert 1e-4 < ((a - b).norm() / a.norm()).item() < 0.03


def test_an_8_bit_head_takes_less_memory_than_a_bf16_one():
    """2048 x 65536 weights: 256 MiB in bf16, 128 in 8 bits.  What the object holds besides is the same but for codes of rows and scales."""
    vocab, d, M = 65536, 2048, 8
    w = torch.zeros(d, vocab, device="cuda", dtype=torch.bfloat16)
    taken = {}
    for which in (tdp.E_LM_HEAD, tdp.E_LM_HEAD_I8):
        torch.cuda.synchronize()
        before = torch.cuda.mem_get_info()[0]
        e = tdp.tdp_ends_create(tdp.EndsConfig(vocab, d, 1e-5, M))
        tdp.tdp_ends_set_weight(e, which, w, tdp.BF16, tdp.DEVICE, d, vocab)
        taken[which] = (before - torch.cuda.mem_get_info()[0]) / 2 ** 20
        tdp.tdp_ends_destroy(e)
    assert taken[tdp.E_LM_HEAD] - taken[tdp.E_LM_HEAD_I8] >= 128 - 16, taken


@pytest.mark.parametrize("first", ["nothing", "a call", "bf16 weights"])
def test_the_forms_of_a_head_in_any_order(first):
    """The bf16 matrix comes back where it was given back, and stays where a call or a captured one has read it."""
    M, vocab, d = 20, 4100, 128
    with Head(vocab, d, M, False) as bf16, Head(vocab, d, M, True) as int8:
        x = bf16.rows(M, 1)
        want, want8 = bf16.logits(x, M)[0], int8.logits(x, M)[0]
    head = Head.__new__(Head)
    head.vocab, head.d, head.weights = vocab, d, bf16.weights
    head.h = tdp.tdp_ends_create(tdp.EndsConfig(vocab, d, 1e-5, M))
    with head:
        tdp.tdp_ends_set_weight(head.h, tdp.E_FINAL_NORM, bf16.gain, tdp.F32, tdp.DEVICE, d, 1)
        graph = None
        if first != "nothing":
            if first == "bf16 weights":
                head.set(False)
            lg, captured = head.logits(x, M)[0], torch.zeros(M, vocab, device="cuda")
            assert torch.equal(lg, want if first == "bf16 weights" else torch.zeros_like(lg))
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
                tdp.tdp_lm_head(head.h, x, M, None, M, captured, None, torch.cuda.current_stream())
        for _ in range(2):
            head.set(True)
            assert torch.equal(head.logits(x, M)[0], want8)
            if graph:                                   # the form that it was captured with
                captured.fill_(7)
                graph.replay()
                torch.cuda.synchronize()
                assert torch.equal(captured, lg)
            head.set(False)
            assert torch.equal(head.logits(x, M)[0], want)
            lg = want


@pytest.mark.parametrize("int8", [False, True])
def test_rows_by_index_and_hidden_states_that_are_not_numbers(int8):
    M, vocab, d = 9, 4100, 128
    with Head(vocab, d, M, int8) as head:
        x = head.rows(40, 2)
        idx = i32([3, 39, 3, 0, 17, 100, -4, 8, 8])          # repeated, and clamped into the rows
        want = [3, 39, 3, 0, 17, 39, 0, 8, 8]
        lp, en, ix, tl, tok = head.logprobs(x, M, None, 3, idx=idx)
        direct = head.logprobs(x[want].contiguous(), M, None, 3)
        for a, b in zip((lp, en, ix, tl, tok), direct):
            assert torch.equal(a, b)
        x[5, 7], x[6, 0] = float("nan"), float("inf")
        lp, en, ix, tl, tok = (a.cpu().numpy() for a in head.logprobs(x[:9].contiguous(), M, [1] * M, 3))
        assert np.isnan(lp[[5, 6]]).all() and np.isnan(en[[5, 6]]).all() and np.isfinite(np.delete(lp, [5, 6])).all()
        assert (ix[5] == -1).all() and tok[5] == 0


# the tile that the batches above leave out, and vocabularies that take it
MORE_BY_TILE = [(65, 50304, 64), (100, 64000, 320), (128, 128256, 64), (3, 4100, 2048)]


def plan_of_int8_head(M, vocab, d):
    padded = -(-vocab // 256) * 256
    return tdp.tdp_gemm_plan_i8(M, vocab, d, False, 2 * min((M + 1) // 2 * 2, 512) * padded)


def test_all_batches_cover_every_kind_of_tile_of_both_heads():
    cases = BY_TILE + MORE_BY_TILE
    bf16, int8 = [plan_of_head(*c) for c in cases], [plan_of_int8_head(*c) for c in cases]
    every = set(range(1, 14)) - {11}      # (11 sums in chunks: of bf16 alone)
    assert {p["tile"] for p in bf16 if p["splits"] == 1 and not p["chunk_k"]} == every
    assert {p["tile"] for p in int8 if p["splits"] == 1} == every
    assert any(p["splits"] > 1 for p in int8) and any(p["splits"] > 1 for p in bf16)
    for vocab in (50304, 64000, 100000, 128256):      # ordinary decode batches
        assert {plan_of_int8_head(M, vocab, 4096)["tile"] for M in (65, 100, 128)} == {2}


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("M,vocab,d", MORE_BY_TILE)
def test_statistics_of_the_other_kinds_of_tiles(M, vocab, d, int8):
    test_statistics_of_every_kind_of_tile(M, vocab, d, int8)


def test_captured_calls_replay_with_new_contents():
    """Both calls in one graph on a stream of their own, replayed with other logits and hidden states, with eager work between."""
    M, vocab, d = 40, 4100, 256
    with Head(vocab, d, M, True) as head:
        x, z = head.rows(M, 1), torch.randn(M, 999, device="cuda")
        targets = i32(np.arange(M))
        lp, en = torch.zeros(M, device="cuda"), torch.zeros(M, device="cuda")
        ix, tl = torch.zeros((M, 4), dtype=torch.int32, device="cuda"), torch.zeros((M, 4), device="cuda")
        lp2, tok = torch.zeros(M, device="cuda"), torch.zeros(M, dtype=torch.int32, device="cuda")
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            s = torch.cuda.current_stream()
            tdp.tdp_logprob_rows(z, tdp.F32, M, 999, 999, targets, 4, lp, en, ix, tl, s)
            tdp.tdp_lm_head_logprobs(head.h, x, M, None, M, targets, 0, tok, lp2, None, None, None, s)
        for seed in range(3):
            x.copy_(head.rows(M, 50 + seed))
            z.copy_(torch.randn(M, 999, device="cuda") * 3)
            graph.replay()
            torch.cuda.synchronize()
            check([a.cpu().numpy() for a in (lp, en, ix, tl)], f64(z), np.arange(M), 4)
            eager = head.logprobs(x, M, np.arange(M), 0)
            torch.cuda.synchronize()
            assert torch.equal(lp2, eager[0]) and torch.equal(tok, eager[4])


def test_a_call_on_another_stream_waits_for_that_streams_work():
    z = torch.randn(64, 32000, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        w = z * 2
        got = call(w, tdp.F32, 64, 32000, 32000, None, 2, s)
    check(got, f64(w), None, 2)


def test_an_8_bit_head_wider_than_its_sums_allow_is_refused():
    """133184 products of 127 * 127 do not fit 32 bits"""
    d = 133184
    e = tdp.tdp_ends_create(tdp.EndsConfig(4, d, 1e-5, 1))
    try:
        w = torch.zeros((d, 4), device="cuda")
        with pytest.raises(tdp.TdpError) as err:
            tdp.tdp_ends_set_weight(e, tdp.E_LM_HEAD_I8, w, tdp.F32, tdp.DEVICE, d, 4)
        assert err.value.code == tdp.EINVAL
        tdp.tdp_ends_set_weight(e, tdp.E_LM_HEAD, w, tdp.F32, tdp.DEVICE, d, 4)
    finally:
        tdp.tdp_ends_destroy(e)
