"""The numbers of a beam search, step by step: every step's logits of every row against an ordinary prefill of that row's own tokens on a stage of
its own (weights and tolerances: search_helpers; what faults would move: test_beam_search_steps_host.py)."""
import numpy as np
import pytest
import torch

from harness import workload as W
from paper_2506_10470_amd import tdp
from paper_2506_10470_amd.engine import BeamSearch
from search_helpers import LOGITS_TOL, LOGITS_TOL_8BIT, SEARCHES, VOCAB, AttentiveStage, histories
from stage_helpers import i32, row_rel_err
from test_gpu_beam_search import Recorder, prompts_of
from test_gpu_ends import Ends

pytestmark = pytest.mark.gpu


def prefilled(st, ends, tokens):
    """Logits behind the last token of every list, from one prefill of them all."""
    lens = [len(t) for t in tokens]
    held = [-(-n // 16) for n in lens]
    tables = np.full((len(tokens), st.max_pages_per_seq), -1, np.int32)
    for r, (n, first) in enumerate(zip(held, np.cumsum([0] + held))):
        tables[r, :n] = first + np.arange(n)
    cu, total = np.concatenate([[0], np.cumsum(lens)]), sum(lens)
    x = torch.empty((total, st.shape.d_model), dtype=torch.bfloat16, device="cuda")
    y, logits = torch.empty_like(x), torch.empty((len(tokens), VOCAB), device="cuda")
    tdp.tdp_embed_tokens(ends.h, i32(np.concatenate(tokens)), total, x)
    tdp.tdp_stage_prefill(st.h, x, i32(cu), i32(tables), len(tokens), total, y)
    tdp.tdp_lm_head(ends.h, y, total, i32(cu[1:] - 1), len(tokens), logits, None)
    torch.cuda.synchronize()
    return logits.double().cpu().numpy()


def check_steps(sh, rec, prompts, longest, kv_scales):
    """The largest row-relative error of all steps' logits, and of how many rows; and that without attention it would be another."""
    steps = histories(prompts, [got[:2] for _, _, _, _, got in rec.selections])[:-1]
    rows, worst, checked = max(map(len, steps)), 0.0, 0
    width = -(-longest // 16)
    with AttentiveStage(tdp, sh, rows * width, rows, rows * longest, rows, width, kv_scales=kv_scales) as st, Ends(sh, VOCAB, rows * longest) as ends:
        for (before, _, _, _, _), tokens in zip(rec.selections, steps):
            real = [r for r, t in enumerate(tokens) if t is not None]
            want = prefilled(st, ends, [tokens[r] for r in real])
            worst = max(worst, row_rel_err(before[0].double().cpu().numpy()[real], want))
            checked += len(real)
            long = [i for i, r in enumerate(real) if len(tokens[r]) > 4]
            if long:
                alone = prefilled(st, ends, [tokens[real[i]][-1:] for i in long])
                assert row_rel_err(alone, want[long]) > 4 * LOGITS_TOL_8BIT
    return worst, checked


@pytest.mark.parametrize("shape,lengths,beams,max_new,end,kv_scales", SEARCHES)
def test_every_step_is_that_of_its_own_history(shape, lengths, beams, max_new, end, kv_scales):
    sh = W.SHAPES[shape]
    prompts, rows, longest = prompts_of(lengths), len(lengths) * beams, max(lengths) + max_new
    pages = sum((n + 15) // 16 for n in lengths) + rows * ((max_new + 15) // 16 + 3)
    rec = Recorder()
    with AttentiveStage(tdp, sh, pages, rows, sum(lengths), len(lengths), -(-longest // 16), kv_scales=kv_scales) as st, Ends(
            sh, VOCAB, max(sum(lengths), rows)) as ends:
        st.poison()
        with BeamSearch(rec, st.h, ends.h, sh.d_model, VOCAB, pages, -(-longest // 16), rows, sum(lengths), len(lengths)) as search:
            search.generate(prompts, beams, max_new, end)
    worst, checked = check_steps(sh, rec, prompts, longest, kv_scales)
    print("%s %s: worst %.2e over %d rows" % (shape, lengths, worst, checked))
    assert checked >= len(lengths) * (1 + beams * (min(max_new, 4) - 1))
    assert worst <= (LOGITS_TOL if kv_scales is None else LOGITS_TOL_8BIT)


@pytest.mark.parametrize("kv_scales", [None, (0.05, 0.04)])
def test_every_step_of_two_stages_is_that_of_one(kv_scales):
    """A pipeline of two stages on a side stream against prefills of the undivided model: a hand-over rounds to bf16 (2^-8 of a hidden state at most),
    for which half of the tolerance comes on top."""
    sh = W.SHAPES["tiny_gqa"]
    prompts, beams, max_new = prompts_of([30, 26]), 3, 20
    rec, layers = Recorder(), sh.n_layers // 2
    stages = [AttentiveStage(tdp, sh.with_layers(layers), 64, 6, 56, 2, 4, layer_offset=i * layers, kv_scales=kv_scales) for i in range(2)]
    with Ends(sh, VOCAB, 56) as ends:
        torch.cuda.synchronize()
        with BeamSearch(rec, [s.h for s in stages], ends.h, sh.d_model, VOCAB, 64, 4, 6, 56, 2, stream=torch.cuda.Stream()) as search:
            search.generate(prompts, beams, max_new)
        torch.cuda.synchronize()
    for s in stages:
        s.close()
    worst, checked = check_steps(sh, rec, prompts, 50, kv_scales)
    print("two stages: worst %.2e over %d rows" % (worst, checked))
    assert checked == 2 + 6 * (max_new - 1)
    assert worst <= 1.5 * (LOGITS_TOL if kv_scales is None else LOGITS_TOL_8BIT)
