"""Operators of decoding with several continuations of a prompt, as measurable calls: the selection over beams and vocabulary, forking and
compacting the block tables of a paged cache with the copies of its pages, and the attention of a batch whose requests share
prefixes.

Every case is one call, or the two that belong together, that a serving engine makes in a step.  Where `own` is false, `run` computes
it in elementary torch operations; where it is true, through `paper_2506_10470_amd.tdp`.  Head layouts and widths are those of the
model shapes in the repository's benchmark and tests.

Pools are in the stage's layout: keys [page][head][bytes of a row / 64][16 slots][64 bytes], values [page][head][channel][16 slots].
"""
import hashlib
import math
import random

import torch

own = False

PAGE = 16
END = 2  # the token that finishes a beam


def listed():
    return [
        # -- selection over beams and vocabulary
        # one request, a toy vocabulary, the step after two beams have finished
        {"name": "select_1x4_1000", "kind": "select", "groups": 1, "beams": 4, "n": 1000, "out": 4, "bf16": False, "finished": True, "masked": False},
        # few requests and a large vocabulary: twice the beams, so that enough are left where some end
        {"name": "select_2x5_128256", "kind": "select", "groups": 2, "beams": 5, "n": 128256, "out": 10, "bf16": False, "finished": False, "masked": False},
        # the benchmark's decode batch as 64 requests, a quarter of them held to a grammar that allows few tokens
        {"name": "select_64x8_32000", "kind": "select", "groups": 64, "beams": 8, "n": 32000, "out": 16, "bf16": False, "finished": False, "masked": True},
        # wide beams, an odd vocabulary, logits in bf16 (many equal ones)
        {"name": "select_33x16_152067_bf16", "kind": "select", "groups": 33, "beams": 16, "n": 152067, "out": 16, "bf16": True, "finished": True, "masked": False},
        # -- block tables: rows continue other rows, and the pages that this makes them copy
        # a beam step of one request
        {"name": "fork_1x4", "kind": "fork", "groups": 1, "beams": 4, "step": True, "prefix": 100, "pages_row": 64, "spare": 200, "heads": 2, "dh": 64, "layers": 2, "kv8": False},
        # a beam step of the benchmark's decode batch behind prompts of a thousand tokens
        {"name": "fork_64x8", "kind": "fork", "groups": 64, "beams": 8, "step": True, "prefix": 1000, "pages_row": 256, "spare": 1500, "heads": 8, "dh": 128, "layers": 2, "kv8": False},
        # prompts just prefilled, each continued 16 times; an 8-bit cache
        {"name": "fork_32_into_512", "kind": "fork", "groups": 32, "beams": 16, "step": False, "prefix": 1700, "pages_row": 300, "spare": 3000, "heads": 8, "dh": 128, "layers": 4, "kv8": True},
        # -- pages moved to the front of the pool
        # what a toy engine does between two batches
        {"name": "compact_5", "kind": "compact", "rows": 5, "length": 120, "pages_row": 16, "used": 0.5, "moves": 32, "heads": 2, "dh": 64, "layers": 2, "kv8": False},
        # a pool after hours of service, a bounded number of moves in one go
        {"name": "compact_256", "kind": "compact", "rows": 256, "length": 900, "pages_row": 128, "used": 0.6, "moves": 2048, "heads": 8, "dh": 64, "layers": 2, "kv8": False},
        # -- attention of a batch that shares prefixes
        # one request's four beams, toy widths
        {"name": "attend_1x4_toy", "kind": "attend", "groups": 1, "rows": 4, "prefix": 100, "suffix": 20, "qh": 8, "heads": 2, "dh": 64, "kv8": False},
        # eight beams of 24 requests, each behind a long prompt, one query head per K/V head; an 8-bit cache
        {"name": "attend_24x8_32h_8bit", "kind": "attend", "groups": 24, "rows": 8, "prefix": 4000, "suffix": 100, "qh": 32, "heads": 32, "dh": 128, "kv8": True},
        # the benchmark's decode batch, all behind one system prompt
        {"name": "attend_1x512_64h8", "kind": "attend", "groups": 1, "rows": 512, "prefix": 2100, "suffix": 300, "qh": 64, "heads": 8, "dh": 128, "kv8": False},
    ]


def draw(rng):
    def spread(lo, hi):  # uniform in the logarithm
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))

    kind = rng.choice(["select", "fork", "compact", "attend", "attend"])
    if kind == "select":
        beams, n = spread(1, 16), spread(300, 152067)
        return {"kind": kind, "groups": spread(1, max(1, min(128, int(8.0e7 / (n * beams))))), "beams": beams, "n": n,
                "out": rng.choice([beams, 2 * beams]), "bf16": rng.random() < 0.4, "finished": rng.random() < 0.4, "masked": rng.random() < 0.3}
    heads, dh = rng.choice([1, 2, 3, 8, 8, 32, 40]), rng.choice([64, 128])
    layout = {"heads": heads, "dh": dh, "kv8": rng.random() < 0.3}
    if kind == "fork":
        step, beams, groups, prefix = rng.random() < 0.7, spread(1, 16), spread(1, 48), spread(1, 2000)
        return {"kind": kind, "groups": groups, "beams": beams, "step": step, "prefix": prefix, "pages_row": (prefix + 200) // PAGE + spread(1, 64),
                "spare": groups * beams * 2 + spread(1, 500), "layers": 1, **layout}
    if kind == "compact":
        rows, length = spread(1, 128), spread(1, 800)
        return {"kind": kind, "rows": rows, "length": length, "pages_row": (length + 15) // PAGE + spread(1, 32), "used": rng.uniform(0.2, 0.95),
                "moves": spread(1, 2000), "layers": 1, **layout}
    group = rng.choice([1, 1, 2, 4, 5, 8, 16])
    while group * heads > 64:
        heads = max(1, heads // 2)
    groups, prefix, suffix = spread(1, 64), spread(1, 8000), spread(1, 400)
    most = 8.0e8 / ((prefix + suffix) * heads * dh * groups)
    return {"kind": kind, "groups": groups, "rows": spread(1, int(max(1, min(most, 512 // groups)))), "prefix": prefix, "suffix": suffix,
            "qh": group * heads, "heads": heads, "dh": dh, "kv8": layout["kv8"]}


# ---- inputs -----------------------------------------------------------------------------------------------------

def number(seed, what):
    return int.from_bytes(hashlib.blake2b(repr((int(seed), what)).encode(), digest_size=7).digest(), "big")


def generator(seed, what):
    return torch.Generator(device="cuda").manual_seed(number(seed, what))


def sizes(case):
    """Random numbers for what a case's lengths and sizes are: the same ones for every seed."""
    return random.Random(number(0, sorted((k, v) for k, v in case.items() if k != "name")))


def normal(seed, what, shape, std=1.0):
    return torch.randn(shape, generator=generator(seed, what), device="cuda").mul_(std)


def whole(seed, what, lo, hi, shape):
    return torch.randint(lo, hi, shape, generator=generator(seed, what), device="cuda", dtype=torch.int32)


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class State:
    """What an engine holds before the call."""


class Handle:
    """An object of the library, given back when nothing refers to it any more."""

    def __init__(self, handle, destroy):
        self.handle, self.destroy = handle, destroy

    def __del__(self):
        self.destroy(self.handle)


class Memory:
    """Device memory of a library's object, for torch.as_tensor, whose tensors keep this and so the object alive."""

    def __init__(self, owner, address, count, kind):
        self.owner = owner
        self.__cuda_array_interface__ = {"shape": (count,), "typestr": kind, "data": (address, False), "version": 2}


def prepare(case, seed):
    S = State()
    S.case, S.kind, S.rng = case, case["kind"], random.Random(number(seed, "host"))
    {"select": prepare_select, "fork": prepare_fork, "compact": prepare_compact, "attend": prepare_attend}[S.kind](S, case, seed)
    if own:
        prepare_own(S, case)
    return S


def prepare_select(S, case, seed):
    S.groups, S.beams, S.n, S.out = case["groups"], case["beams"], case["n"], case["out"]
    rows = S.groups * S.beams
    S.logits = normal(seed, "logits", (rows, S.n), 2.5)
    S.logits.view(S.groups, S.beams, S.n)[:, :, whole(seed, "likely", 0, S.n, (8,)).long()] += 8.0
    if case["masked"]:  # every fourth request may go on with at most 24 tokens
        allowed = whole(seed, "allowed", 0, S.n, ((S.groups + 3) // 4, 24)).long()
        keep = torch.zeros(allowed.shape[0], S.n, dtype=torch.bool, device="cuda").scatter_(1, allowed, True)
        S.logits.view(S.groups, S.beams, S.n)[::4].masked_fill_(~keep[:, None, :], -math.inf)
    # beams come in order of their scores, a few tenths to a few nats apart, after some ten tokens
    S.scores = (-normal(seed, "gaps", (S.groups, S.beams)).abs().cumsum(1) - 12.0 - normal(seed, "level", (S.groups, 1), 4.0).abs()).reshape(-1)
    S.finished = None
    if case["finished"]:
        S.finished = (whole(seed, "finished", 0, 100, (rows,)) < 25).int()
        S.finished[:: 2 * S.beams] = 1  # the best beam of every second request
    if case["bf16"]:
        S.logits = S.logits.to(torch.bfloat16)


def pools(S, case, seed, count):
    """Keys and values of `count` pages, one after the other for every layer."""
    shape = (case["layers"], count, case["heads"] * PAGE * case["dh"])
    S.count, S.kv8 = count, case["kv8"]
    if S.kv8:
        S.k, S.v = ((whole(seed, what, 0, 1 << 31, (shape[0], count, shape[2] // 4))).view(torch.uint8) for what in ("keys", "values"))
    else:
        S.k, S.v = (normal(seed, what, shape).to(torch.bfloat16) for what in ("keys", "values"))


def fork_lengths(case):
    """(tokens of the prompt, tokens in all) of every request, the same for its beams; and the pages that they hold."""
    rng, lengths = sizes(case), []
    for _ in range(case["groups"]):
        prefix = max(1, int(case["prefix"] * rng.uniform(0.6, 1.0)))
        lengths.append((prefix, prefix + (rng.randint(1, 150) if case["step"] else 0)))
    rows = case["beams"] if case["step"] else 1
    return lengths, sum(prefix // PAGE + rows * ((n + 15) // PAGE - prefix // PAGE) for prefix, n in lengths)


def going_on(case):
    """How many of a request's beams go on in a step: six of ten, some of them twice and more often."""
    return max(1, math.ceil(0.6 * case["beams"])) if case["step"] else 1


def prepare_fork(S, case, seed):
    groups, beams = case["groups"], case["beams"]
    rng = S.rng
    per_group = beams if case["step"] else 1
    S.n_src, S.n_dst, width = groups * per_group, groups * beams, case["pages_row"]
    lengths, need = fork_lengths(case)
    parents = []
    for g in range(groups):
        alive = rng.sample(range(per_group), going_on(case))
        chosen = alive + [rng.choice(alive) for _ in range(beams - len(alive))]
        rng.shuffle(chosen)
        parents += [g * per_group + p for p in chosen]
    count = need + case["spare"]
    ids = rng.sample(range(count), need)
    refs, rows, lens = [0] * count, [], []
    for prefix, length in lengths:
        shared = [ids.pop() for _ in range(prefix // PAGE)]
        for _ in range(per_group):
            row = shared + [ids.pop() for _ in range((length + 15) // PAGE - len(shared))]
            for p in row:
                refs[p] += 1
            rows.append(row + [-1] * (width - len(row)))
            lens.append(length)
    S.tables, S.lens, S.refs, S.parents, S.width = i32(rows), i32(lens), i32(refs), i32(parents), width
    pools(S, case, seed, count)


def compact_lengths(case):
    """The rows' tokens, and how many pages each has in common with the first row; pages in rows, pages that somebody else holds, and all."""
    rng = sizes(case)
    lens = [rng.randint(0 if i % 7 == 3 else 1, case["length"]) for i in range(case["rows"])]
    held = [(n + 15) // PAGE for n in lens]
    shared = [min(h, held[0]) // 2 if i % 3 == 1 else 0 for i, h in enumerate(held)]
    need = sum(held) - sum(shared)
    pinned = max(1, need // 50)
    return lens, held, shared, need, pinned, int((need + pinned) / case["used"]) + 1


def prepare_compact(S, case, seed):
    rng, S.n_rows, S.width, S.moves = S.rng, case["rows"], case["pages_row"], case["moves"]
    lens, held, shared, need, pinned, count = compact_lengths(case)
    ids = rng.sample(range(count), need + pinned)
    refs, rows = [0] * count, []
    for i, h in enumerate(held):
        row = (rows[0][:shared[i]] if i else []) + [ids.pop() for _ in range(h - shared[i])]
        for p in row:
            refs[p] += 1
        rows.append(row + [-1] * (S.width - h))
    for p in ids:
        refs[p] += 1
    for i in range(0, S.n_rows, 11):  # and the first page of some rows is held by others as well
        if held[i]:
            refs[rows[i][0]] += 1
    S.tables, S.lens, S.refs = i32(rows), i32(lens), i32(refs)
    pools(S, case, seed, count)


def attend_lengths(case):
    """Where the groups begin and end, the rows' tokens, and the whole pages that a row's group shares."""
    rng, starts, lens, shared = sizes(case), [0], [], []
    for _ in range(case["groups"]):
        size = case["rows"] if case["groups"] == 1 else max(1, int(round(case["rows"] * rng.uniform(0.7, 1.0))))
        prefix = max(1, int(case["prefix"] * rng.uniform(0.5, 1.0)))
        starts.append(starts[-1] + size)
        shared += [prefix // PAGE] * size
        lens += [prefix + rng.randint(1, case["suffix"]) for _ in range(size)]
    return starts, lens, shared


def prepare_attend(S, case, seed):
    S.groups, S.qh, S.heads, S.dh = case["groups"], case["qh"], case["heads"], case["dh"]
    starts, lens, shared = attend_lengths(case)
    S.batch = starts[-1]
    S.width = (case["prefix"] + case["suffix"] + 15) // PAGE
    held = [(n + 15) // PAGE for n in lens]
    need = sum(shared[b] for b in starts[:-1]) + sum(h - s for h, s in zip(held, shared))
    count = need + max(1, need // 8)
    ids = torch.randperm(count, generator=generator(seed, "pages"), device="cuda").tolist()
    rows = []
    for g in range(S.groups):
        common = [ids.pop() for _ in range(shared[starts[g]])]
        rows += [common + [ids.pop() for _ in range(held[b] - len(common))] + [-1] * (S.width - held[b]) for b in range(starts[g], starts[g + 1])]
    S.tables, S.lens, S.starts = i32(rows), i32(lens), i32(starts)
    S.count, S.kv8 = count, case["kv8"]
    shape = (1, count, S.heads * PAGE * S.dh)
    S.k_scale, S.v_scale = (0.02, 0.015) if S.kv8 else (1.0, 1.0)
    if S.kv8:  # codes of numbers, no NaN among them
        S.k, S.v = (normal(seed, what, shape, 1.0 / scale).clamp_(-440, 440).to(torch.float8_e4m3fn).view(torch.uint8)
                    for what, scale in (("keys", S.k_scale), ("values", S.v_scale)))
    else:
        S.k, S.v = (normal(seed, what, shape).to(torch.bfloat16) for what in ("keys", "values"))
    S.q = normal(seed, "queries", (S.batch, S.qh, S.dh), 1.5).to(torch.bfloat16)


def prepare_own(S, case):
    from paper_2506_10470_amd import tdp
    S.tdp = tdp
    if S.kind == "select":
        rows = S.groups * S.beams
        S.owner = Handle(tdp.tdp_beams_create(tdp.BeamsConfig(rows, S.out)), tdp.tdp_beams_destroy)
        S.parent, S.token, S.ended = (torch.empty((S.groups, S.out), dtype=torch.int32, device="cuda") for _ in range(3))
        S.score = torch.empty((S.groups, S.out), device="cuda")
        return
    layers = 1 if S.kind == "attend" else case["layers"]
    batch = S.batch if S.kind == "attend" else 1
    heads, dh, qh = case["heads"], case["dh"], case.get("qh", case["heads"])
    stage = tdp.tdp_stage_create(tdp.StageConfig(
        n_layers=layers, d_model=64, n_q_heads=qh, n_kv_heads=heads, head_dim=dh, d_ff=64, rms_eps=1e-5, rope_base=10000.0, page_size=PAGE,
        num_pages=S.count, max_batch=batch, max_tokens=0, max_seqs=0, max_pages_per_seq=S.width,
        kv_dtype=tdp.KV_FP8_E4M3 if S.kv8 else tdp.KV_BF16, k_scale=S.k_scale if S.kind == "attend" else 0.0,
        v_scale=S.v_scale if S.kind == "attend" else 0.0, decode_micro_batches=0))
    S.owner = Handle(stage, tdp.tdp_stage_destroy)
    ks, vs = [], []
    for layer in range(layers):  # the stage's pools instead of the plain ones
        k, v, size = tdp.tdp_stage_kv_pool(stage, layer)
        for views, address, plain in ((ks, k, S.k), (vs, v, S.v)):
            view = torch.as_tensor(Memory(S.owner, address, size, "|u1"), device="cuda")
            view = (view if S.kv8 else view.view(torch.bfloat16)).view(plain[layer].shape)
            view.copy_(plain[layer])
            views.append(view)
    S.k, S.v = ks, vs
    if S.kind == "attend":
        S.answer = torch.empty_like(S.q)
        return
    rows = S.n_rows if S.kind == "compact" else max(S.n_src, S.n_dst)
    S.pages = Handle(tdp.tdp_pages_create(tdp.PagesConfig(S.count, rows, S.width)), tdp.tdp_pages_destroy)
    S.new_refs = torch.empty_like(S.refs)
    S.status = torch.empty(4, dtype=torch.int32, device="cuda")
    S.new_tables = torch.empty((rows if S.kind == "compact" else S.n_dst, S.width), dtype=torch.int32, device="cuda")
    if S.kind == "fork":
        S.new_lens = torch.empty(S.n_dst, dtype=torch.int32, device="cuda")
    S.pairs = torch.empty((S.moves if S.kind == "compact" else S.n_dst, 2), dtype=torch.int32, device="cuda")


# ---- the calls --------------------------------------------------------------------------------------------------

def run(S):
    if own:
        return run_own(S)
    return {"select": plain_select, "fork": plain_fork, "compact": plain_compact, "attend": plain_attend}[S.kind](S)


def run_own(S):
    tdp = S.tdp
    if S.kind == "select":
        tdp.tdp_beams_select(S.owner.handle, S.logits, tdp.BF16 if S.logits.dtype == torch.bfloat16 else tdp.F32, S.groups, S.beams, S.n, S.n,
                             S.scores, S.finished, END, S.out, S.parent, S.token, S.score, S.ended)
        return {"parent": S.parent, "token": S.token, "score": S.score, "finished": S.ended}
    if S.kind == "attend":
        tdp.tdp_stage_attend(S.owner.handle, 0, S.q, S.lens, S.tables, S.batch, S.starts, S.groups, S.answer)
        return S.answer
    if S.kind == "fork":
        tdp.tdp_pages_fork(S.pages.handle, S.parents, S.tables, S.lens, S.n_src, None, 1, S.n_dst, S.refs, S.new_refs, S.new_tables, S.new_lens,
                           S.pairs, S.status)
    else:
        tdp.tdp_pages_compact(S.pages.handle, S.tables, S.lens, S.n_rows, S.moves, S.refs, S.new_refs, S.new_tables, S.pairs, S.status)
    tdp.tdp_stage_kv_copy_pages(S.owner.handle, S.pairs, S.pairs.shape[0])
    got = {"tables": S.new_tables, "refs": S.new_refs, "pairs": S.pairs, "status": S.status, "keys": S.k, "values": S.v}
    return {**got, "lens": S.new_lens} if S.kind == "fork" else got


def plain_select(S):
    z = S.logits.float().view(S.groups, S.beams, S.n)
    if S.finished is not None:  # a finished beam goes on with the end token alone, which costs nothing
        only = torch.where(torch.arange(S.n, device="cuda") == END, 0.0, -math.inf)
        z = torch.where((S.finished != 0).view(S.groups, S.beams, 1), only, z)
    # the order of candidates is decided in 64 bits
    top = z.amax(2, keepdim=True).double()
    log_total = torch.log(torch.exp(z.double() - top).sum(2, keepdim=True)) + top
    # the likeliest tokens of every beam, by one whole number each: the logit's bits made monotone, then the lower index
    bits = (z + 0.0).view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32) + torch.arange(S.n - 1, -1, -1, device="cuda")
    each = min(S.out, S.n)
    index = order.topk(each, 2).indices
    candidate = (S.scores.double().view(S.groups, S.beams, 1) + (z.gather(2, index).double() - log_total)).view(S.groups, -1)
    candidate = torch.where(candidate > -math.inf, candidate, -math.inf)  # (NaN: no candidate)
    value, place = candidate.sort(dim=1, descending=True, stable=True)  # of equal ones the lower beam, then the lower token
    value, place = value[:, :S.out], place[:, :S.out]
    some = value > -math.inf
    token = torch.where(some, index.view(S.groups, -1).gather(1, place), -1)
    first = torch.arange(S.groups, device="cuda")[:, None] * S.beams
    parent = torch.where(some, place // each + first, -1)
    return {"parent": parent.int(), "token": token.int(), "score": value.float(), "finished": (token == END).int()}


def copied(pool, pairs):
    real = pairs[pairs[:, 0] >= 0].long()
    pool[:, real[:, 1]] = pool[:, real[:, 0]]
    return [pool[layer] for layer in range(pool.shape[0])]


def plain_fork(S, add=1):
    parents = S.parents.long()
    old_len, column = S.lens.long(), torch.arange(S.width, device="cuda")
    length = old_len[parents]
    new_len, shared, held = length + add, length // PAGE, (length + PAGE - 1) // PAGE
    row = torch.arange(S.n_dst, device="cuda")
    first = torch.full((S.n_src,), S.n_dst, device="cuda").scatter_reduce(0, parents, row, "amin")
    keeps = first[parents] == row
    partial = length % PAGE != 0
    page = S.tables[parents, shared.clamp(max=S.width - 1)].long().clamp(min=0)
    copies = partial & ~(keeps & (S.refs[page] == 1))
    fresh_from = torch.where(copies, shared, held)
    new_held = (new_len + PAGE - 1) // PAGE
    fresh = new_held - fresh_from
    before = fresh.cumsum(0) - fresh
    free = torch.nonzero(S.refs == 0)[:, 0]
    rank = before[:, None] + column[None] - fresh_from[:, None]
    is_fresh = (column >= fresh_from[:, None]) & (column < new_held[:, None])
    given = free[rank.clamp(0, max(0, free.numel() - 1))]
    old = S.tables[parents].long()
    tables = torch.where(is_fresh, given, torch.where(column < new_held[:, None], old, -1))
    pairs = torch.where(copies[:, None], torch.stack([page, free[before.clamp(max=max(0, free.numel() - 1))]], 1), -1)
    # references: every table entry is one
    gone = S.tables[column < ((old_len + PAGE - 1) // PAGE)[:, None]].long()
    come = tables[column < new_held[:, None]]
    refs = S.refs.long().index_add(0, come, torch.ones_like(come)).index_add(0, gone, -torch.ones_like(gone))
    status = torch.stack([torch.zeros_like(row[0]), torch.zeros_like(row[0]), fresh.sum(), (S.refs == 0).sum()])
    pairs = pairs.int()
    return {"tables": tables.int(), "refs": refs.int(), "pairs": pairs, "status": status.int(), "keys": copied(S.k, pairs),
            "values": copied(S.v, pairs), "lens": new_len.int()}


def plain_compact(S):
    column = torch.arange(S.width, device="cuda")
    held = column < ((S.lens.long() + PAGE - 1) // PAGE)[:, None]
    pages = S.tables[held].long()
    counted = torch.zeros_like(S.refs).index_add(0, pages, torch.ones_like(pages, dtype=torch.int32))
    free = torch.nonzero(S.refs == 0)[:, 0][:S.moves]
    movable = torch.nonzero((S.refs > 0) & (counted == S.refs))[:, 0].flip(0)[:S.moves]
    most = min(free.numel(), movable.numel())
    free, movable = free[:most], movable[:most]
    goes = free < movable
    free, movable = free[goes], movable[goes]
    to = torch.arange(S.count, device="cuda").index_copy(0, movable, free)
    tables = torch.where(held, to[S.tables.long().clamp(min=0)].int(), -1)
    refs = S.refs.index_copy(0, free, S.refs[movable]).index_copy(0, movable, torch.zeros_like(movable, dtype=torch.int32))
    pairs = torch.full((S.moves, 2), -1, dtype=torch.int32, device="cuda")
    pairs[:free.numel()] = torch.stack([movable, free], 1).int()
    zero = torch.zeros((), dtype=torch.int64, device="cuda")
    status = torch.stack([zero, zero, zero + free.numel(), (S.refs > 0).sum()])
    return {"tables": tables, "refs": refs, "pairs": pairs, "status": status.int(), "keys": copied(S.k, pairs), "values": copied(S.v, pairs)}


def e4m3_values():
    """The value of every 8-bit code (a NaN counts as zero here: no input holds one)."""
    code = torch.arange(256, device="cuda")
    exponent, mantissa = (code >> 3) & 15, (code & 7).float()
    value = torch.where(exponent == 0, mantissa * 2.0 ** -9, torch.exp2(exponent.float() - 10) * (8 + mantissa))
    return torch.where((code & 127) == 127, 0.0, torch.where(code >= 128, -value, value))


def plain_attend(S):
    pages, at = S.tables.long().clamp(min=0), torch.arange(S.width * PAGE, device="cuda")
    k, v = S.k[0][pages.view(-1)], S.v[0][pages.view(-1)]
    if S.kv8:
        value = e4m3_values()
        k, v = value[k.long()] * S.k_scale, value[v.long()] * S.v_scale
    piece = 64 // (1 if S.kv8 else 2)
    # [row][head][position][channel] of both
    k = k.float().view(S.batch, S.width, S.heads, S.dh // piece, PAGE, piece).permute(0, 2, 1, 4, 3, 5).reshape(S.batch, S.heads, -1, S.dh)
    v = v.float().view(S.batch, S.width, S.heads, S.dh, PAGE).permute(0, 2, 1, 4, 3).reshape(S.batch, S.heads, -1, S.dh)
    q = S.q.float().view(S.batch, S.heads, S.qh // S.heads, S.dh)
    score = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(S.dh)
    score = torch.where(at < S.lens[:, None, None, None], score, -math.inf)
    e = torch.exp(score - score.amax(3, keepdim=True))
    o = torch.matmul(e, v) / e.sum(3, keepdim=True)
    return o.reshape(S.q.shape).to(torch.bfloat16)


# ---- what a pass has to do, and its result in 64 bits -----------------------------------------------------------

def work(case):
    if case["kind"] == "select":
        rows = case["groups"] * case["beams"]
        left = 0.75 if case["finished"] else 1.0  # (of a finished beam no logit is needed)
        return {"bytes": left * rows * case["n"] * (2 if case["bf16"] else 4) + rows * 8 + case["groups"] * case["out"] * 16,
                "flops": left * 4.0 * rows * case["n"]}
    size = 1 if case["kv8"] else 2
    if case["kind"] == "attend":
        starts, lens, shared = attend_lengths(case)
        once = sum(shared[b] for b in starts[:-1]) * PAGE
        own_tokens = sum(lens) - sum(shared) * PAGE
        return {"bytes": 2.0 * case["heads"] * case["dh"] * size * (once + own_tokens) + len(lens) * case["qh"] * case["dh"] * 4,
                "flops": 4.0 * sum(lens) * case["qh"] * case["dh"]}
    page = 2.0 * case["heads"] * case["dh"] * PAGE * size * case["layers"]  # keys and values
    if case["kind"] == "fork":
        lengths, need = fork_lengths(case)
        held = sum((n + 15) // PAGE for _, n in lengths)
        rows_in = case["beams"] if case["step"] else 1
        copies = (case["beams"] - going_on(case)) * sum(n % PAGE != 0 for _, n in lengths)
        return {"bytes": 4.0 * held * (rows_in + case["beams"]) + 8.0 * (need + case["spare"]) + 2 * page * copies, "flops": 0.0}
    _, held, _, need, pinned, count = compact_lengths(case)
    moves = min(case["moves"], need * (1 - case["used"]))  # (the free ids among as many as there are pages in use)
    return {"bytes": 8.0 * sum(held) + 8.0 * count + 2 * page * moves, "flops": 0.0}


def exact(case, seed):
    if case["kind"] in ("fork", "compact"):
        return None  # whole numbers and copies
    S = prepare({**case}, seed)
    if S.kind == "select":
        z = S.logits.double().view(S.groups, S.beams, S.n)
        c = z - torch.logsumexp(z, 2, keepdim=True) + S.scores.double().view(S.groups, S.beams)[:, :, None]
        if S.finished is not None:
            done = S.finished.view(S.groups, S.beams).bool()
            c[done] = -math.inf
            c[:, :, END][done] = S.scores.double().view(S.groups, S.beams)[done]
        return {"parent": None, "token": None, "score": c.view(S.groups, -1).topk(S.out, 1).values, "finished": None}
    if S.batch * S.width * PAGE * S.qh * S.dh > 2.5e11:
        return None
    table = torch.arange(256, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).double()
    out = torch.empty((S.batch, S.qh, S.dh), dtype=torch.float64, device="cuda")
    lens, piece = S.lens.tolist(), 64 if S.kv8 else 32
    for b in range(S.batch):
        n = lens[b]
        page = S.tables[b, :(n + 15) // PAGE].long()
        k, v = S.k[0].index_select(0, page), S.v[0].index_select(0, page)
        k, v = (table[k.int()] * S.k_scale, table[v.int()] * S.v_scale) if S.kv8 else (k.double(), v.double())
        k = k.view(-1, S.heads, S.dh // piece, PAGE, piece).permute(1, 0, 3, 2, 4).reshape(S.heads, -1, S.dh)[:, :n]
        v = v.view(-1, S.heads, S.dh, PAGE).permute(1, 0, 3, 2).reshape(S.heads, -1, S.dh)[:, :n]
        q = S.q[b].double().view(S.heads, -1, S.dh)
        p = torch.softmax(q.bmm(k.transpose(1, 2).contiguous()) * S.dh ** -0.5, -1)
        out[b] = p.bmm(v.contiguous()).view(S.qh, S.dh)
    return out
