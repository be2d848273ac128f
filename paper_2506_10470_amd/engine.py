"""A worker that runs what the scheduling library decides: the executor side of tdp_simulate_exec.

The paper's engine tells each worker which batch to run in which phase (Sec. 3.2); the decisions are
those of Sec. 3.3 - 3.5 (libtdp_sched.so).  This module is the worker for ONE GPU: it owns the page
allocation (the engine's job, Sec. 3.2.1), turns each event of the schedule into calls of the stage
library (token embedding -> tdp_stage_prefill / tdp_stage_decode -> final norm + vocabulary
projection + greedy selection) and keeps every request's tokens.  The pipeline clock of the
schedule still comes from the profiles handed to the scheduler; the work itself is done by the HIP
kernels, on the stream the caller names, and so are the copies in front of them and behind them: ids and
tables up, answers down.  BeamSearch, beside the worker, searches with several continuations of every prompt, whose
tables the device itself forks.  Host logic only: no arithmetic of the method lives here.
"""
from __future__ import annotations

import functools
from typing import Dict, List, Optional, Sequence, Tuple

import numpy as np
import torch

PAGE = 16


class OutOfPages(RuntimeError):
    pass


def _on_own_stream(method):
    """The method with the worker's stream as the current one, behind what the caller's current stream holds: torch's copies are then
    ordered with the kernels, and memory that it takes and gives back is reused behind them."""
    @functools.wraps(method)
    def run(self, *args):
        callers = torch.cuda.current_stream()
        if callers != self.torch_stream:
            self.torch_stream.wait_stream(callers)
        with torch.cuda.stream(self.torch_stream):
            return method(self, *args)
    return run


class StageWorker:
    """Executes prefill / decode / release events on a stage (tdp_stage) and a pair of pipeline ends
    (tdp_ends) that the caller created and loaded.  `prompts[i]` are request i's prompt token ids.
    `stage` may also be a sequence of stage handles: the stages of a pipeline held by one GPU, run one
    after the other on every batch (hidden states handed from each to the next as bf16, the pipeline's
    hand-over format, Sec. 2.2.3); they share the block tables, every stage owning its own pools of
    `num_pages` pages."""

    def __init__(self, tdp, stage: int, ends: int, d_model: int, num_pages: int, max_pages_per_seq: int,
                 max_batch: int, max_tokens: int, max_seqs: int, prompts: Sequence[Sequence[int]], stream=None,
                 check_tables: bool = False, logprobs: Optional[int] = None):
        """stream: a torch stream or its address (none: the current one); all of the worker's work is ordered on it, behind
        what the caller's current stream holds at each event.  logprobs: the log-probability of every
        generated token goes to self.logprobs[i] (beside self.generated[i]), and of the `logprobs` likeliest tokens in its place
        (0: none) as (token, log-probability) pairs to self.top[i].  check_tables: validate every call's block tables on the GPU
        first (tdp_stage_check_*): one synchronisation per call, for runs that test the allocator rather than the throughput."""
        self.tdp, self.ends = tdp, ends
        self.stages = [stage] if isinstance(stage, int) else list(stage)
        self.stage = self.stages[0]
        self.d_model = d_model
        self.max_pps, self.max_batch, self.max_tokens, self.max_seqs = max_pages_per_seq, max_batch, max_tokens, max_seqs
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        self.free_pages: List[int] = list(range(num_pages - 1, -1, -1))
        self.num_pages = num_pages
        self.check_tables = check_tables
        self.pages: Dict[int, List[int]] = {}
        self.prompts = [list(map(int, p)) for p in prompts]
        self.generated: List[List[int]] = [[] for _ in prompts]
        if logprobs is not None and not 0 <= logprobs <= tdp.MAX_TOP:
            raise ValueError("logprobs must be 0 .. %d" % tdp.MAX_TOP)
        self.n_top = logprobs
        self.logprobs: List[List[float]] = [[] for _ in prompts]
        self.top: List[List[List[Tuple[int, float]]]] = [[] for _ in prompts]
        self.torch_stream = (self.stream if isinstance(self.stream, torch.cuda.Stream)
                             else torch.cuda.ExternalStream(getattr(self.stream, "cuda_stream", self.stream)))
        self._buffers(max(max_batch, max_tokens, 1), max(max_batch, max_seqs, 1))
        self.stats = {"prefill_batches": 0, "prefill_tokens": 0, "decode_steps": 0, "decode_tokens": 0,
                      "released": 0, "evicted": 0, "min_free_pages": num_pages}

    @_on_own_stream
    def _buffers(self, rows: int, answers: int) -> None:
        self.hidden = torch.empty((rows, self.d_model), dtype=torch.bfloat16, device="cuda")
        self.hidden_out = torch.empty_like(self.hidden)
        self.next_tok = torch.empty(answers, dtype=torch.int32, device="cuda")
        if self.n_top is not None:
            self.tok_logprob = torch.empty(answers, dtype=torch.float32, device="cuda")
            self.top_index = torch.empty((answers, self.n_top), dtype=torch.int32, device="cuda")
            self.top_logprob = torch.empty((answers, self.n_top), dtype=torch.float32, device="cuda")

    # ---- pages
    def _take(self, n: int) -> List[int]:
        if n > len(self.free_pages):
            raise OutOfPages("need %d pages, %d free" % (n, len(self.free_pages)))
        got = [self.free_pages.pop() for _ in range(n)]
        self.stats["min_free_pages"] = min(self.stats["min_free_pages"], len(self.free_pages))
        return got

    def _table(self, ids: Sequence[int]) -> torch.Tensor:
        t = np.zeros((len(ids), self.max_pps), dtype=np.int32)
        for k, rid in enumerate(ids):
            p = self.pages[rid]
            t[k, :len(p)] = p
        return torch.from_numpy(t).cuda()

    @staticmethod
    def _i32(a) -> torch.Tensor:
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()

    # ---- behind the last stage
    def _answer(self, ids: Sequence[int], hidden: torch.Tensor, row_index) -> None:
        """The next token of every request of a batch, from its row of the last hidden states."""
        tdp, n = self.tdp, len(ids)
        if self.n_top is None:
            tdp.tdp_lm_head(self.ends, hidden, hidden.shape[0], row_index, n, None, self.next_tok[:n], self.stream)
        else:
            some = self.n_top > 0
            tdp.tdp_lm_head_logprobs(self.ends, hidden, hidden.shape[0], row_index, n, None, self.n_top, self.next_tok[:n],
                                     self.tok_logprob[:n], None, self.top_index if some else None, self.top_logprob if some else None,
                                     self.stream)
        tokens = self.next_tok[:n].cpu().tolist()
        for rid, t in zip(ids, tokens):
            self.generated[rid].append(int(t))
        if self.n_top is not None:
            index, values = self.top_index[:n].cpu().tolist(), self.top_logprob[:n].cpu().tolist()
            for rid, lp, i, v in zip(ids, self.tok_logprob[:n].cpu().tolist(), index, values):
                self.logprobs[rid].append(lp)
                self.top[rid].append(list(zip(i, v)))

    # ---- the three events
    @_on_own_stream
    def prefill(self, ids: List[int], lens: List[int]) -> None:
        n, total = len(ids), int(sum(lens))
        if n > self.max_seqs or total > self.max_tokens:
            raise ValueError("prefill batch of %d prompts / %d tokens exceeds the stage's limits" % (n, total))
        toks: List[int] = []
        for rid, L in zip(ids, lens):
            seq = self.prompts[rid] + self.generated[rid]
            if len(seq) != L:
                raise ValueError("request %d: schedule says %d tokens, worker holds %d" % (rid, L, len(seq)))
            if rid in self.pages:
                raise ValueError("request %d is prefilled while it still holds pages" % rid)
            if (L + PAGE - 1) // PAGE > self.max_pps:
                raise ValueError("request %d does not fit a block-table row" % rid)
            self.pages[rid] = self._take((L + PAGE - 1) // PAGE)
            toks += seq
        cu = np.zeros(n + 1, dtype=np.int32)
        cu[1:] = np.cumsum(lens)
        tdp = self.tdp
        x, y = self.hidden[:total], self.hidden_out[:total]
        cu_dev, table = self._i32(cu), self._table(ids)
        if self.check_tables:
            tdp.tdp_stage_check_prefill(self.stage, cu_dev, table, n, total, self.stream)
        tdp.tdp_embed_tokens(self.ends, self._i32(toks), total, x, self.stream)
        for st in self.stages:
            tdp.tdp_stage_prefill(st, x, cu_dev, table, n, total, y, self.stream)
            x, y = y, x
        y = x
        self._answer(ids, y, self._i32(cu[1:] - 1))
        self.stats["prefill_batches"] += 1
        self.stats["prefill_tokens"] += total

    @_on_own_stream
    def decode(self, batch: int, ids: List[int], contexts: List[int]) -> None:
        n = len(ids)
        if n == 0:
            return
        if n > self.max_batch:
            raise ValueError("decode batch of %d exceeds the stage's max_batch %d" % (n, self.max_batch))
        for rid, ctx in zip(ids, contexts):
            if ctx != len(self.prompts[rid]) + len(self.generated[rid]) - 1:
                raise ValueError("request %d: schedule says %d cached tokens, worker holds %d" % (
                    rid, ctx, len(self.prompts[rid]) + len(self.generated[rid]) - 1))
            if ctx // PAGE >= self.max_pps:
                raise ValueError("request %d outgrew its block-table row" % rid)
            if ctx // PAGE >= len(self.pages[rid]):
                self.pages[rid] += self._take(1)
        tdp = self.tdp
        x, y = self.hidden[:n], self.hidden_out[:n]
        ctx_dev, table = self._i32(contexts), self._table(ids)
        if self.check_tables:
            tdp.tdp_stage_check_decode(self.stage, ctx_dev, table, n, self.stream)
        tdp.tdp_embed_tokens(self.ends, self._i32([self.generated[rid][-1] for rid in ids]), n, x, self.stream)
        for st in self.stages:
            tdp.tdp_stage_decode(st, x, ctx_dev, table, n, y, self.stream)
            x, y = y, x
        y = x
        self._answer(ids, y, None)
        self.stats["decode_steps"] += 1
        self.stats["decode_tokens"] += n

    def release(self, ids: List[int], reason: int) -> None:
        for rid in ids:
            self.free_pages.extend(reversed(self.pages.pop(rid)))
        self.stats["released" if reason == 0 else "evicted"] += len(ids)

    # ---- the run
    def run(self, sched, cfg, requests: Sequence[Tuple[int, int, int]], decode_profile, prefill_profile,
            events_cap: int = 0):
        """requests[i] = (input_len, output_len, predict_len) with input_len = len(prompts[i]).  Returns
        (SimResult, events) of the scheduling library; the tokens are in self.generated."""
        if len(requests) != len(self.prompts) or any(r[0] != len(p) for r, p in zip(requests, self.prompts)):
            raise ValueError("requests and prompts disagree")
        return sched.tdp_simulate_exec(cfg, requests, decode_profile, prefill_profile, prefill=self.prefill,
                                       decode=self.decode, release=self.release, events_cap=events_cap)


class BeamSearch:
    """Beam search on a stage (or the stages of a pipeline held by one GPU) and a pair of pipeline ends: prompts are prefilled once, their
    rows fork into `beams` rows, and every step decodes all beams with their shared prefixes read once, ranks the continuations of a
    request's beams over the whole vocabulary, and forks the block tables accordingly.  Choices, tables and page copies stay on the
    device: the host reads nothing between the steps but, every `stop_every` steps, whether all beams have ended.
    It owns the pages of the stages while it runs.  Row b of a step is beam b % beams of request b // beams."""

    def __init__(self, tdp, stage, ends: int, d_model: int, vocab_size: int, num_pages: int, max_pages_per_seq: int, max_batch: int,
                 max_tokens: int, max_seqs: int, stream=None):
        self.tdp, self.ends = tdp, ends
        self.stages = [stage] if isinstance(stage, int) else list(stage)
        self.d_model, self.vocab_size, self.num_pages, self.max_pps = d_model, vocab_size, num_pages, max_pages_per_seq
        self.max_batch, self.max_tokens, self.max_seqs = max_batch, max_tokens, max_seqs
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        self.torch_stream = (self.stream if isinstance(self.stream, torch.cuda.Stream)
                             else torch.cuda.ExternalStream(getattr(self.stream, "cuda_stream", self.stream)))
        rows = max(max_batch, max_seqs, 1)
        self.pages = self.select = None
        try:
            self.pages = tdp.tdp_pages_create(tdp.PagesConfig(num_pages, rows, max_pages_per_seq))
            self.select = tdp.tdp_beams_create(tdp.BeamsConfig(rows, tdp.MAX_TOP))
        except BaseException:
            self.close()
            raise

    def close(self) -> None:
        """Gives the library's objects back."""
        if self.pages:
            self.tdp.tdp_pages_destroy(self.pages)
        if self.select:
            self.tdp.tdp_beams_destroy(self.select)
        self.pages = self.select = None

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    def generate(self, prompts: Sequence[Sequence[int]], beams: int, max_new: int, end_token: int = -1,
                 stop_every: int = 8) -> List[List[Tuple[List[int], float]]]:
        """For every prompt its beams, best first: (generated tokens, sum of their log-probabilities).  A beam that chose end_token keeps it as
        its last token.  Beams that never had a continuation of their own (logits without a distribution, or with fewer tokens above minus infinity
        than beams) are left out."""
        n = len(prompts)
        if n < 1 or any(len(p) < 1 for p in prompts):
            raise ValueError("every prompt needs a token")
        if not 1 <= beams <= min(self.tdp.MAX_BEAMS, self.tdp.MAX_TOP, self.vocab_size) or max_new < 1 or stop_every < 1:
            raise ValueError("beams must be 1 .. %d and within the vocabulary, max_new and stop_every at least 1" % self.tdp.MAX_TOP)
        if not -1 <= end_token < self.vocab_size:
            raise ValueError("end_token must be a token, or -1 for none")
        total, rows = sum(map(len, prompts)), n * beams
        if n > self.max_seqs or total > self.max_tokens or rows > self.max_batch:
            raise ValueError("%d prompts, %d tokens, %d beams exceed the stage's limits" % (n, total, rows))
        longest = max(map(len, prompts)) + max_new
        if longest > PAGE * self.max_pps:
            raise ValueError("%d tokens do not fit a block-table row" % longest)
        # pages of the prompts, those that beams have of their own, and those that a step's new rows take before the old ones give theirs back
        needed = sum(-(-len(p) // PAGE) for p in prompts) + rows * (-(-max_new // PAGE) + 1) + 2 * rows
        if needed > self.num_pages:
            raise OutOfPages("up to %d pages are needed, there are %d" % (needed, self.num_pages))
        return self._generate([list(map(int, p)) for p in prompts], beams, max_new, end_token, stop_every)

    @_on_own_stream
    def _generate(self, prompts, beams, max_new, end_token, stop_every):
        tdp, n, rows = self.tdp, len(prompts), len(prompts) * beams
        total = sum(map(len, prompts))
        i32 = StageWorker._i32

        def ints(*shape):  # (zeros: whatever has not been written names a page that there is)
            return torch.zeros(shape, dtype=torch.int32, device="cuda")
        refs = torch.zeros(self.num_pages, dtype=torch.int32, device="cuda")
        states = [(ints(max(rows, n), self.max_pps), ints(max(rows, n))) for _ in range(2)]  # tables and lengths, before and behind a fork
        copies, status = ints(max(rows, n), 2), ints(max_new + 1, 4)
        parents, tokens, ended = ints(max_new, rows), ints(max_new, rows), ints(max_new, rows)
        scores = [torch.empty(rows, dtype=torch.float32, device="cuda") for _ in range(2)]
        x = torch.empty((max(total, rows), self.d_model), dtype=torch.bfloat16, device="cuda")
        y = torch.empty_like(x)
        logits = torch.empty((rows, self.vocab_size), dtype=torch.float32, device="cuda")

        # the prompts
        lens = [len(p) for p in prompts]
        cu = np.zeros(n + 1, dtype=np.int32)
        cu[1:] = np.cumsum(lens)
        cu_dev, (tables, table_lens) = i32(cu), states[0]
        tdp.tdp_pages_fork(self.pages, None, None, None, 0, i32(lens), 0, n, refs, refs, tables, table_lens, copies, status[0], self.stream)
        tdp.tdp_embed_tokens(self.ends, i32(sum(prompts, [])), total, x, self.stream)
        for st in self.stages:
            tdp.tdp_stage_prefill(st, x, cu_dev, tables, n, total, y, self.stream)
            x, y = y, x
        tdp.tdp_lm_head(self.ends, x, total, i32(cu[1:] - 1), n, logits, None, self.stream)
        scores[0][:n] = 0
        tdp.tdp_beams_select(self.select, logits, tdp.F32, n, 1, self.vocab_size, self.vocab_size, scores[0], None, end_token, beams, parents[0], tokens[0],
                             scores[1], ended[0], self.stream)
        # A row's length is that of the tokens that its pages have room for: with the one that is decoded next.
        groups, step, n_src = i32(np.arange(n + 1) * beams), 0, n
        while step + 1 < max_new:
            (tables, table_lens), (new_tables, new_lens) = states[step % 2], states[(step + 1) % 2]
            tdp.tdp_pages_fork(self.pages, parents[step], tables, table_lens, n_src, None, 1, rows, refs, refs, new_tables, new_lens, copies,
                               status[step + 1], self.stream)
            for st in self.stages:
                tdp.tdp_stage_kv_copy_pages(st, copies, rows, self.stream)
            if (step + 1) % stop_every == 0 and bool((status[:, :2] != 0).any() | (ended[step] != 0).all()):
                break
            ctx = new_lens - 1
            tdp.tdp_embed_tokens(self.ends, tokens[step], rows, x, self.stream)
            for st in self.stages:
                tdp.tdp_stage_decode_shared(st, x, ctx, new_tables, rows, groups, n, y, self.stream)
                x, y = y, x
            tdp.tdp_lm_head(self.ends, x, rows, None, rows, logits, None, self.stream)
            step, n_src = step + 1, rows
            tdp.tdp_beams_select(self.select, logits, tdp.F32, n, beams, self.vocab_size, self.vocab_size, scores[step % 2],
                                 ended[step - 1] if end_token >= 0 else None, end_token, beams, parents[step], tokens[step], scores[(step + 1) % 2],
                                 ended[step], self.stream)
        if bool((status[:, :2] != 0).any()):  # (the fork that ended the search among them)
            raise OutOfPages("a fork of the block tables found no page")
        parents, tokens, final = parents[:step + 1].cpu().tolist(), tokens[:step + 1].cpu().tolist(), scores[(step + 1) % 2].cpu().tolist()
        answers = []
        for g in range(n):
            answers.append([])
            for row in range(g * beams, (g + 1) * beams):
                found, at = [], row
                for s in range(step, -1, -1):
                    if at < 0 or tokens[s][at] < 0:
                        break
                    found.append(tokens[s][at])
                    at = parents[s][at]
                else:
                    found.reverse()
                    if end_token in found:
                        found = found[:found.index(end_token) + 1]
                    answers[g].append((found, final[row]))
        return answers
