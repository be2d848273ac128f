"""Beam search through the engine: attention over shared prefixes, selection, forked tables and page copies as one loop on the device.

Every decision of a run is recorded and checked against the oracles on what it was made from (selection on the logits that the head gave,
tables on the tables before them); the numbers are checked by scoring each answer again from nothing, prompt and tokens in one ordinary
prefill, whose log-probabilities add up to the score that the search gave it."""
import numpy as np
import pytest
import torch

from harness import workload as W
from oracle import beams_oracle as B
from oracle import pages_oracle as P
from paper_2506_10470_amd import tdp
from paper_2506_10470_amd.engine import BeamSearch, OutOfPages
from stage_helpers import Stage, i32
from test_gpu_beams import check
from test_gpu_ends import Ends

pytestmark = pytest.mark.gpu
VOCAB = 512


class Recorder:
    """The binding, with what the search's decisions were made from and what they were."""

    def __init__(self):
        self.selections, self.forks = [], []

    def __getattr__(self, name):
        return getattr(tdp, name)

    def tdp_beams_select(self, h, logits, dtype, groups, beams, n, ld, scores, finished, end, n_out, parent, token, score, ended, stream):
        rows = groups * beams
        before = logits[:rows].clone(), scores[:rows].cpu().numpy(), None if finished is None else finished[:rows].cpu().numpy()
        tdp.tdp_beams_select(h, logits, dtype, groups, beams, n, ld, scores, finished, end, n_out, parent, token, score, ended, stream)
        torch.cuda.synchronize()
        got = [t[:groups * n_out].view(groups, n_out).cpu().numpy() for t in (parent, token, score, ended)]
        self.selections.append((before, beams, n_out, end, got))

    def tdp_pages_fork(self, h, parents, src_tables, src_lens, n_src, add, add_all, n_dst, refs_in, refs_out, tables, lens, copies, status, stream):
        torch.cuda.synchronize()
        before = ([-1] * n_dst if parents is None else parents[:n_dst].tolist(), [] if n_src == 0 else src_tables[:n_src].tolist(),
                  [] if n_src == 0 else src_lens[:n_src].tolist(), [add_all] * n_dst if add is None else add[:n_dst].tolist(), refs_in.tolist())
        tdp.tdp_pages_fork(h, parents, src_tables, src_lens, n_src, add, add_all, n_dst, refs_in, refs_out, tables, lens, copies, status, stream)
        torch.cuda.synchronize()
        width = tables.shape[1]
        want = P.fork(*before, width)
        assert (tables[:n_dst].tolist(), lens[:n_dst].tolist(), refs_out.tolist(), [tuple(c) for c in copies[:n_dst].tolist()],
                tuple(status.tolist())) == want
        self.forks.append((before, want))


def prompts_of(lengths):
    return [list(map(int, W.token_ids(VOCAB, n, 900 + i))) for i, n in enumerate(lengths)]


def scored_again(sh, ends, tokens, first, kv_scales):
    """Log-probabilities of tokens[first:], from one prefill of all of them on a stage of its own; and the largest logit."""
    n = len(tokens)
    with Stage(tdp, sh, (n + 15) // 16, 1, n, 1, (n + 15) // 16, kv_scales=kv_scales) as st:
        x = torch.empty((n, sh.d_model), dtype=torch.bfloat16, device="cuda")
        y = torch.empty_like(x)
        tdp.tdp_embed_tokens(ends.h, i32(tokens), n, x)
        tdp.tdp_stage_prefill(st.h, x, i32([0, n]), i32(np.arange((n + 15) // 16)[None]), 1, n, y)
        logits = torch.empty((n, VOCAB), device="cuda")
        tdp.tdp_lm_head(ends.h, y, n, None, n, logits, None)
        torch.cuda.synchronize()
        z = logits.double()
        lp = torch.log_softmax(z, 1)[torch.arange(n - 1), torch.tensor(tokens[1:], device="cuda")]
        return lp[first - 1:].cpu().numpy(), z.abs().max().item()


@pytest.mark.parametrize("shape,lengths,beams,max_new,end,kv_scales", [
    ("tiny", [5], 4, 20, -1, None), ("tiny_gqa", [40, 16, 33], 3, 36, -1, None), ("tiny_gqa", [100, 7], 8, 18, 13, (0.05, 0.04)),
    ("tiny_h128", [64, 65], 5, 17, -1, None), ("tiny_mqa", [300], 2, 5, 7, None), ("tiny", [1, 2, 3], 1, 12, -1, None)])
def test_every_decision_of_a_search_and_its_scores(shape, lengths, beams, max_new, end, kv_scales):
    sh = W.SHAPES[shape]
    prompts, rows = prompts_of(lengths), len(lengths) * beams
    width = (max(lengths) + max_new + 15) // 16
    pages = sum((n + 15) // 16 for n in lengths) + rows * ((max_new + 15) // 16 + 3)
    rec = Recorder()
    with Stage(tdp, sh, pages, rows, sum(lengths), len(lengths), width, kv_scales=kv_scales) as st, Ends(sh, VOCAB, max(sum(lengths), rows, max(lengths) + max_new)) as ends:
        st.poison()
        with BeamSearch(rec, st.h, ends.h, sh.d_model, VOCAB, pages, width, rows, sum(lengths), len(lengths)) as search:
            found = search.generate(prompts, beams, max_new, end)
            steps = len(rec.selections)
            assert steps == max_new or end >= 0
            for (logits, scores, finished), w, n_out, e, got in rec.selections:
                check(got, logits, scores, w, n_out, finished, e)
            # what one step gives is what the next one takes
            for a, b in zip(rec.selections, rec.selections[1:]):
                assert np.array_equal(a[4][2].reshape(-1), b[0][1])
                assert b[0][2] is None or np.array_equal(a[4][3].reshape(-1), b[0][2])
            for (a, want), (b, _) in zip(rec.forks, rec.forks[1:]):
                assert b[1] == want[0] and b[2] == want[1] and b[4] == want[2]
            assert [f[0][0] for f in rec.forks[1:]] == [s[4][0].reshape(-1).tolist() for s in rec.selections[:len(rec.forks) - 1]]
            for g, answers in enumerate(found):
                assert len(answers) == beams and [s for _, s in answers] == sorted((s for _, s in answers), reverse=True)
                assert len({tuple(t) for t, _ in answers}) == beams
                for tokens, score in answers:
                    assert len(tokens) == steps or tokens[-1] == end
                    # the relative 2e-2 of a row that the stage's tests allow its hidden states, and so its logits, on either side
                    lp, largest = scored_again(sh, ends, prompts[g] + tokens, lengths[g], kv_scales)
                    assert abs(lp.sum() - score) <= 2 * 2e-2 * largest * len(tokens), (g, score, lp.sum())
            # and again, from the pages that the run before left
            again = search.generate(prompts, beams, max_new, end)
            assert again == found


def test_a_pipeline_of_two_stages_on_a_side_stream():
    sh = W.SHAPES["tiny_gqa"]
    prompts, beams, max_new = prompts_of([30, 50]), 3, 20
    answers = []
    for parts in (1, 2):
        layers = sh.n_layers // parts
        stages = [Stage(tdp, sh.with_layers(layers), 64, 6, 80, 2, 5, layer_offset=i * layers) for i in range(parts)]
        with Ends(sh, VOCAB, 80) as ends:
            torch.cuda.synchronize()
            side = torch.cuda.Stream()
            with BeamSearch(tdp, [s.h for s in stages], ends.h, sh.d_model, VOCAB, 64, 5, 6, 80, 2, stream=side) as search:
                answers.append(search.generate(prompts, beams, max_new))
            torch.cuda.synchronize()
        for s in stages:
            s.close()
    one, two = answers
    # (a hand-over rounds to bf16: scores agree as far as that goes, beams may end in another order)
    for a, b in zip(one, two):
        assert len(a) == len(b) == beams and abs(a[0][1] - b[0][1]) <= 2 * 2e-2 * 10 * max_new


def test_a_search_ends_when_all_beams_have():
    """With an end token that every beam chooses at once nothing is decoded behind the first check."""
    sh = W.SHAPES["tiny"]
    with Stage(tdp, sh, 64, 4, 20, 1, 8) as st, Ends(sh, VOCAB, 20) as ends:
        rec = Recorder()
        with BeamSearch(rec, st.h, ends.h, sh.d_model, VOCAB, 64, 8, 4, 20, 1) as search:
            best = search.generate(prompts_of([9]), 1, 3)[0][0][0]
            rec.selections.clear()
            found = search.generate(prompts_of([9]), 1, 60, end_token=best[1], stop_every=4)
            assert found[0][0][0] == best[:best.index(best[1]) + 1]
            assert len(rec.selections) <= 4


def test_refusals():
    sh = W.SHAPES["tiny"]
    with Stage(tdp, sh, 16, 4, 40, 2, 4) as st, Ends(sh, VOCAB, 40) as ends:
        with BeamSearch(tdp, st.h, ends.h, sh.d_model, VOCAB, 16, 4, 4, 40, 2) as search:
            for prompts, beams, new, kw in [([], 1, 1, {}), ([[]], 1, 1, {}), ([[1]], 0, 1, {}), ([[1]], 33, 1, {}), ([[1]], 1, 0, {}), ([[1]] * 3, 1, 1, {}),
                                            ([[1] * 41], 1, 1, {}), ([[1]], 5, 1, {}), ([[1] * 40], 1, 25, {}), ([[1]], 1, 1, dict(end_token=VOCAB)),
                                            ([[1]], 1, 1, dict(end_token=-2)), ([[1]], 1, 1, dict(stop_every=0))]:
                with pytest.raises(ValueError):
                    search.generate(prompts, beams, new, **kw)
            with pytest.raises(OutOfPages):
                search.generate([[1] * 20, [2] * 20], 2, 40)
            assert len(search.generate([[1] * 20], 1, 16)[0]) == 1


@pytest.mark.parametrize("stop_every", [1, 3, 100])
def test_a_fork_that_finds_no_page_is_an_error(stop_every):
    """Also where it is the one that ends the search.  (generate() asks for enough pages beforehand; what is behind that check is called here.)"""
    sh = W.SHAPES["tiny"]
    with Stage(tdp, sh, 16, 4, 40, 2, 4) as st, Ends(sh, VOCAB, 40) as ends:
        with BeamSearch(tdp, st.h, ends.h, sh.d_model, VOCAB, 5, 4, 4, 40, 2) as search:
            with pytest.raises(OutOfPages):     # four beams behind 31 tokens: the prompt's two pages, and three more where four are needed
                search._generate([[1] * 31], 4, 6, -1, stop_every)
            assert len(search._generate([[1] * 20], 1, 6, -1, stop_every)[0]) == 1
