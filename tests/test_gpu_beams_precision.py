"""Beam selection where the order hangs on a candidate's last bits: rows held to one token, rows that differ by a constant, and candidates that fp32
cannot tell apart (inputs and bound: beams_helpers)."""
import numpy as np
import pytest
import torch

from beams_helpers import CLOSE, bound, close_rows, misplaced
from oracle import beams_oracle as B
from test_gpu_beams import INF, Beams

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", CLOSE)
@pytest.mark.parametrize("seed", [1, 2])
def test_candidates_that_fp32_cannot_tell_apart(case, seed):
    groups, beams, n = case[:3]
    z, scores = close_rows(seed, *case)
    logits = torch.from_numpy(z).cuda()
    if case[-1]:
        assert torch.equal(logits.bfloat16().float(), logits)
        logits = logits.bfloat16()
    with Beams(groups * beams, 32) as b:
        parent, token, score, _ = b.select(logits, scores.tolist(), beams, min(beams, 32))
    c = B.candidates(z, scores, None, -1)
    assert misplaced(c, bound(z), beams, parent, token)[0] == 0
    # and the score that it gives is the candidate's, rounded once (2^-24 of it)
    want = c[parent, token]
    assert (np.abs(score - want) <= bound(z)[parent] + (2.0 ** -24 + 2.0 ** -50) * np.abs(want)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("masked", [-INF, "lowest"])
@pytest.mark.parametrize("n", [1, 2, 77, 5000, 40001, 300007])
def test_a_row_held_to_one_token_costs_nothing(n, masked, dtype):
    """Scores come out as they went in, and equal ones go to the lower beam, whatever the logit, wherever the token."""
    rng = np.random.default_rng(n)
    beams = 32
    low = -INF if masked == -INF else torch.finfo(dtype).min
    z = torch.full((2 * beams, n), low, dtype=dtype, device="cuda")
    at = torch.from_numpy(rng.integers(0, n, 2 * beams)).cuda()
    value = torch.from_numpy(rng.choice([0.0, 1.0, -7.3, 1e-6, 0.1, 88.8, -1234.5, 3e5, 1e30, 2.0 ** -130, 15.625], 2 * beams)).to(dtype).cuda()
    z[torch.arange(2 * beams), at] = value
    tokens = at.view(2, beams).tolist()
    with Beams(2 * beams, beams) as b:
        for s in (0.0, -1.0, -40.1, -1e-3):
            parent, token, score, _ = b.select(z, [s] * (2 * beams), beams, beams)
            assert parent.tolist() == [list(range(beams)), list(range(beams, 2 * beams))] and token.tolist() == tokens
            assert (score == np.float32(s)).all()
        # a finished beam, whose score is its own by definition, among them; and scores that are not all equal
        finished = rng.integers(0, 2, 2 * beams).tolist()
        scores = rng.choice([-0.5, -0.25, -3.0], 2 * beams).astype(np.float32)
        parent, token, score, _ = b.select(z, scores.tolist(), beams, beams, finished, 0)
        for g in range(2):
            order = sorted(range(g * beams, (g + 1) * beams), key=lambda r: (-scores[r], r))
            assert parent[g].tolist() == order and score[g].tolist() == scores[order].tolist()
            assert token[g].tolist() == [0 if finished[r] else int(at[r]) for r in order]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,tokens", [(2, 2)] + [(n, tokens) for n in (9, 1000, 33003, 200001) for tokens in (2, 3)])
def test_rows_that_differ_by_a_constant_are_equal(n, tokens, dtype):
    """Two or three tokens left, the same distances between their logits in every beam, the logits themselves anything: of equal candidates the lower
    beam comes first."""
    rng = np.random.default_rng(n + tokens)
    beams, apart = 10, [0.0, 0.5, 2.0][:tokens]
    at = np.sort(rng.permutation(n)[:tokens])
    base = [0.0, 1.0, -8.5, 24.0, -3.5, 12.0, 0.5, -31.0, 7.0, 28.0]      # (and what is subtracted: values of bf16)
    z = torch.full((beams, n), -INF, dtype=dtype, device="cuda")
    for j, d in enumerate(apart):
        z[:, int(at[j])] = (torch.tensor(base) - d).to(dtype).cuda()
    with Beams(beams, 30) as b:
        for s in (0.0, -3.3, -100.7):
            parent, token, score, _ = b.select(z, [s] * beams, beams, tokens * beams)
            assert parent.tolist() == [list(range(beams)) * tokens]
            assert token.tolist() == [[int(t) for t in at for _ in range(beams)]]
            assert (score.reshape(tokens, beams) == score.reshape(tokens, beams)[:, :1]).all()
        # every logit there is, the same distances
        z = (torch.randint(-16, 16, (1, n), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda") * 0.5 + torch.tensor(base, device="cuda")[:, None]).to(dtype)
        parent, token, _, _ = b.select(z, [-1.5] * beams, beams, beams)
        best = torch.argmax((z[0] == z[0].max()).int()).item()
        assert parent.tolist() == [list(range(beams))] or (z[0] == z[0].max()).sum() > 1
        if (z[0] == z[0].max()).sum() == 1:
            assert token.tolist() == [[best] * beams]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [3, 3001, 50000])
def test_equal_logits_cost_the_logarithm_of_their_number(n, dtype):
    """Also where they are the type's lowest value, beside which the logarithm would be lost, or its highest."""
    for value in (torch.finfo(dtype).min, -1e30, -5.0, 0.0, 1e30, torch.finfo(dtype).max):
        z = torch.full((3, n), value, dtype=dtype, device="cuda")
        with Beams(3, 2) as b:
            parent, token, score, _ = b.select(z, [-1.0, -0.5, -1.0], 3, 2)
        assert parent.tolist() == [[1, 1]] and token.tolist() == [[0, 1]]
        assert (score == np.float32(-0.5 - np.log(n))).all()


def test_a_term_is_off_by_no_more_than_stated():
    """Two tokens d apart: the likelier one's candidate is -ln(1 + e^-d), whose own rounding to fp32 (2^-24 of it) hides little of the term's error of
    (1 + d) 2^-23 where d is large; and the bound as it stands where it is small."""
    rng = np.random.default_rng(1)
    rows = 1 << 16
    d = np.concatenate([rng.uniform(0, 2, rows // 4), rng.uniform(2, 20, rows // 2), rng.uniform(20, 86, rows // 4)]).astype(np.float32)
    top = rng.choice([0.0, 1.0, -5.5, 20.0], rows).astype(np.float32)
    z = np.stack([top, top - d], 1)
    with Beams(rows, 1) as b:
        parent, token, score, _ = b.select(torch.from_numpy(z).cuda(), [0.0] * rows, 1, 1)
    x = z.astype(np.float64)
    apart = x[:, 0] - x[:, 1]
    assert (apart > 0).sum() > rows - 10 and (token[apart > 0] == 0).all() and (parent[:, 0] == np.arange(rows)).all()
    want = -np.log1p(np.exp(-apart))
    off = np.abs(score[:, 0] - want)
    # (in 64 bits: 1 + e^-d is rounded by 2^-53 of itself, 1 to 2, and its logarithm is that much off, whatever is left of it)
    allowed = 2.0 ** -23 * (1 + apart) * np.exp(-apart) / (1 + np.exp(-apart)) + (2.0 ** -24 + 2.0 ** -50) * np.abs(want) + 2.0 ** -52
    for low, high in ((0, 0.5), (0.5, 2), (2, 8), (8, 20), (20, 87)):
        some = (apart >= low) & (apart < high)
        print("%g to %g apart: at most %.2f of what is allowed" % (low, high, (off / allowed)[some].max()))
    assert (off <= allowed).all()
