"""Decode steps with groups at ctx_lens that do not fit their block-table rows: tdp_stage_decode_shared takes such a length as the nearest that
the row can hold, as tdp_stage_decode does, so the step is to the bit the one with those lengths, and the rows beside are what they were."""
import numpy as np
import pytest
import torch

from harness import workload as W
from harness.runner import Stage, i32
from paper_2506_10470_amd import tdp

pytestmark = pytest.mark.gpu
INT_MAX, INT_MIN = 2 ** 31 - 1, -2 ** 31


def filled(sh, tables, width, kv_scales=None):
    """A stage whose rows hold tokens in every slot of their pages."""
    B = len(tables)
    total = B * width * 16
    st = Stage(tdp, sh, B * width, B, 0, 0, width, kv_scales=kv_scales)
    full = i32(np.arange(B + 1) * width * 16)
    for l in range(sh.n_layers):
        k, v = (W.kv_packed(sh, l, w, total, 7, device="cuda") for w in "kv")
        tdp.tdp_stage_kv_import(st.h, l, k, v, full, i32(tables), B, total)
    return st


def step(st, x, ctx, tables, starts):
    out = torch.full_like(x, float("nan"))
    ctx = i32(np.asarray(ctx, np.int64).astype(np.int32))
    tdp.tdp_stage_decode_shared(st.h, x, ctx, i32(tables), len(tables), i32(starts) if starts else None, max(0, len(starts) - 1), out)
    torch.cuda.synchronize()
    return out.view(torch.int16)


def pools(st):
    torch.cuda.synchronize()
    return [t.view(torch.int16).clone() for l in range(st.shape.n_layers) for t in st.pools(l)]


@pytest.mark.parametrize("shape", ["tiny_gqa", "tiny_h128"])
@pytest.mark.parametrize("span", [0, 256, 1024])
@pytest.mark.parametrize("starts", [[], [0, 5], [0, 2, 5], [0, 1, 2, 3, 4, 5]])
def test_a_length_outside_its_row_is_the_nearest_inside(shape, span, starts):
    sh, width = W.SHAPES[shape].with_layers(2), 40
    good = [0, 300, 639, 17, 511]
    for bad in ([INT_MAX, 640, 100000, -5, INT_MIN], [20, INT_MAX, 639, 300, INT_MAX], [INT_MAX] * 5, [INT_MAX - 1, 639, INT_MIN, INT_MAX - 15, 1]):
        nearest = [min(max(n, 0), width * 16 - 1) for n in bad]
        tables = np.random.default_rng(3).permutation(5 * width).reshape(5, width)
        x = W.hidden_states(sh, 5, 1, device="cuda")
        results = []
        for first in (nearest, bad):
            with filled(sh, tables, width) as st:
                tdp.tdp_stage_set_decode_span(st.h, span)
                results.append((step(st, x, first, tables, starts), pools(st), step(st, x, good, tables, starts), pools(st)))
        (out, kv, later, kv_later), (got, got_kv, got_later, got_kv_later) = results
        assert not torch.isnan(out.view(torch.bfloat16).float()).any()
        assert torch.equal(got, out) and torch.equal(got_later, later)
        assert all(torch.equal(a, b) for a, b in zip(got_kv + got_kv_later, kv + kv_later))


@pytest.mark.parametrize("kv_scales", [None, (0.05, 0.04)])
def test_rows_behind_a_shared_prefix_beside_a_length_outside_its_row(kv_scales):
    """Groups whose rows begin with the same pages: the row of the bad length is part of its group, or stands alone."""
    sh, width, rows = W.SHAPES["tiny_gqa"].with_layers(2), 8, 7
    own = np.random.default_rng(4).permutation(rows * width).reshape(rows, width)
    tables = own.copy()
    tables[1:4, :3] = tables[0, :3]
    tables[5:7, :2] = tables[4, :2]
    x = W.hidden_states(sh, rows, 2, device="cuda")
    for starts in ([0, 4, 7], [0, 7], [0, 3, 4, 7]):
        for bad in ([50, 60, 70, INT_MAX, 40, INT_MAX, 127], [INT_MAX, 60, 70, 49, INT_MAX, 41, 90], [INT_MAX] * 7):
            outs = []
            for ctx in ([min(n, width * 16 - 1) for n in bad], bad):
                with filled(sh, own, width, kv_scales) as st:
                    outs.append(step(st, x, ctx, tables, starts))
            assert not torch.isnan(outs[0].view(torch.bfloat16).float()).any()
            assert torch.equal(*outs), (starts, bad)


def test_more_rows_than_the_plan_holds_at_once():
    """Every third of 1100 rows has a length that its row cannot hold."""
    sh, width, rows = W.SHAPES["tiny"].with_layers(1), 2, 1100
    tables = np.random.default_rng(5).permutation(rows * width).reshape(rows, width)
    bad = [(INT_MAX, 5, 31)[b % 3] for b in range(rows)]
    x = W.hidden_states(sh, rows, 3, device="cuda")
    for starts in ([], [0, rows], list(range(rows + 1))):
        outs = []
        for ctx in ([min(n, width * 16 - 1) for n in bad], bad):
            with filled(sh, tables, width) as st:
                outs.append(step(st, x, ctx, tables, starts))
        assert not torch.isnan(outs[0].view(torch.bfloat16).float()).any()
        assert torch.equal(*outs)
