"""The worker with log-probabilities, and with a vocabulary projection in 8 bits, through a whole schedule (prefills, decode steps,
evictions): the decisions and the page accounting are those of any run, every token comes with its log-probability and its alternatives,
and scoring a finished request's tokens with the stage's own prefill gives the numbers that its generation gave."""
import numpy as np
import pytest
import torch

from harness import workload as W
from oracle import sched_oracle as S
from paper_2506_10470_amd import tdp
from paper_2506_10470_amd import tdp_sched as L
from paper_2506_10470_amd.engine import StageWorker
from stage_helpers import Stage, i32
from test_gpu_engine import DEC, PRE, VOCAB, make_requests
from test_gpu_ends import Ends

pytestmark = pytest.mark.gpu


def set_int8(ends, sh):
    tdp.tdp_ends_set_weight(ends.h, tdp.E_LM_HEAD_I8, ends.head, tdp.BF16, tdp.DEVICE, sh.d_model, VOCAB)


@pytest.mark.parametrize("int8,n_top", [(False, None), (False, 0), (False, 3), (True, None), (True, 5)])
def test_a_schedule_with_log_probabilities(int8, n_top):
    sh = W.SHAPES["tiny_gqa"]
    reqs, prompts = make_requests(24, 5)
    capacity, budget = 600, 128
    max_len = max(r[0] + r[1] for r in reqs) + 1
    max_pps = (max_len + 15) // 16 + 1
    num_pages = (capacity + 15) // 16 + len(reqs)
    rows = max(budget, max_len, len(reqs))
    with Stage(tdp, sh, num_pages, len(reqs), rows, len(reqs), max_pps) as st, Ends(sh, VOCAB, rows) as ends:
        if int8:
            set_int8(ends, sh)
        st.poison()
        w = StageWorker(tdp, st.h, ends.h, sh.d_model, num_pages, max_pps, len(reqs), rows, len(reqs), prompts, check_tables=True,
                        logprobs=n_top)
        res, ev = w.run(L, L.SimConfig(2, capacity, budget, 1, 1, 1, 1), reqs, DEC, PRE, events_cap=1 << 20)
        torch.cuda.synchronize()
        ref = S.simulate(reqs, S.SimConfig(2, capacity, budget, True, True, True, True), DEC, PRE)
        assert [(k, a, b) for k, _, a, b in ev] == [(k, a, b) for k, _, a, b in ref.events]
        assert [len(g) for g in w.generated] == [r[1] for r in reqs]
        if n_top is None:
            assert not any(w.logprobs) and not any(w.top)
            return
        assert [len(g) for g in w.logprobs] == [r[1] for r in reqs] == [len(g) for g in w.top]
        for g, lps, tops in zip(w.generated, w.logprobs, w.top):
            for token, lp, top in zip(g, lps, tops):
                assert len(top) == n_top and lp <= 0
                values = [v for _, v in top]
                assert values == sorted(values, reverse=True)
                if n_top:
                    assert top[0][0] == token and len({t for t, _ in top}) == n_top
                    assert abs(top[0][1] - lp) <= 4 * 2.0 ** -24 * (1 + abs(lp))     # -ln s, and 0 - ln s
        # a request alone, scored: its prompt and tokens prefilled in one go, every position's next token its target.  Prefill and
        # decode round the hidden states differently (bf16 between layers): the relative 2e-2 that the stage's own tests allow them.
        i = int(np.argmax([r[1] for r in reqs]))
        tokens = list(map(int, prompts[i])) + w.generated[i]
        n = len(tokens)
        x = torch.empty((n, sh.d_model), dtype=torch.bfloat16, device="cuda")
        y = torch.empty_like(x)
        tdp.tdp_embed_tokens(ends.h, i32(tokens), n, x)
        table = i32(np.arange(max_pps)[None])
        tdp.tdp_stage_prefill(st.h, x, i32([0, n]), table, 1, n, y)
        scores = torch.empty(n, device="cuda")
        tdp.tdp_lm_head_logprobs(ends.h, y, n, None, n, i32(tokens[1:] + [-1]), 0, None, scores, None, None, None)
        logits = torch.empty((n, VOCAB), device="cuda")
        tdp.tdp_lm_head(ends.h, y, n, None, n, logits, None)
        torch.cuda.synchronize()
        scores = scores.cpu().numpy()
        assert np.isneginf(scores[-1])
        first = len(prompts[i]) - 1
        slack = 2 * 2e-2 * logits.abs().max().item()
        assert np.abs(scores[first:-1] - w.logprobs[i]).max() <= slack


def test_the_worker_refuses_more_alternatives_than_there_can_be():
    with pytest.raises(ValueError):
        StageWorker(tdp, 1, 1, 64, 4, 4, 4, 4, 4, [[1]], logprobs=tdp.MAX_TOP + 1)


def run_on(stream, sh, reqs, prompts, busy):
    """A schedule with log-probabilities on `stream` (None: the current one), each event behind `busy` passes over 1 GiB on it."""
    capacity, budget = 600, 128
    max_len = max(r[0] + r[1] for r in reqs) + 1
    max_pps = (max_len + 15) // 16 + 1
    num_pages = (capacity + 15) // 16 + len(reqs)
    rows = max(budget, max_len, len(reqs))
    with Stage(tdp, sh, num_pages, len(reqs), rows, len(reqs), max_pps) as st, Ends(sh, VOCAB, rows) as ends:
        st.poison()
        big = torch.zeros(1 << 28, device="cuda")
        torch.cuda.synchronize()
        w = StageWorker(tdp, st.h, ends.h, sh.d_model, num_pages, max_pps, len(reqs), rows, len(reqs), prompts, stream=stream, logprobs=3)
        late = []

        def behind_other_work(event):
            def call(*args):
                with torch.cuda.stream(w.torch_stream):
                    for _ in range(busy):
                        big.add_(1)
                event(*args)
                late.append(torch.cuda.current_stream() == before)
            return call
        before = torch.cuda.current_stream()
        w.prefill, w.decode = behind_other_work(w.prefill), behind_other_work(w.decode)
        w.run(L, L.SimConfig(2, capacity, budget, 1, 1, 1, 1), reqs, DEC, PRE, events_cap=1 << 20)
        torch.cuda.synchronize()
        assert late and all(late)          # (the caller's current stream is what it was)
        return w.generated, w.logprobs, w.top


def test_a_worker_on_a_stream_of_its_own_gives_the_same_answers():
    """The same calls on the same shapes: the same bits.  Ids, tables and answers are copied while the worker's stream is milliseconds
    behind the caller's, and the caller's current stream, on which copies would not wait, is another."""
    sh = W.SHAPES["tiny_gqa"]
    reqs, prompts = make_requests(12, 9)
    want = run_on(None, sh, reqs, prompts, 0)
    side = torch.cuda.Stream()
    assert run_on(side, sh, reqs, prompts, 4) == want
    assert run_on(side.cuda_stream, sh, reqs, prompts, 4) == want          # by its address
