"""Outputs that overlap inputs or one another, where workgroups would read what others have written: refused, as far as a call does not allow
them, and nothing is written."""
import pytest
import torch

from harness import workload as W
from paper_2506_10470_amd import tdp
from stage_helpers import Stage, i32

pytestmark = pytest.mark.gpu


class Memory:
    """Arrays one behind the other in one piece of memory, so that overlaps of any size can be named."""

    def __init__(self, **sizes):
        self.sizes, self.at, n = sizes, {}, 0
        for name, size in sizes.items():
            self.at[name] = n
            n += size
        self.all = torch.zeros(n, dtype=torch.int32, device="cuda")
        self.base = self.all.data_ptr()

    def ptr(self, name, over=None, end=False):
        """The address of an array; or one that overlaps array `over` with its last number, or (end) with its first."""
        if over is None:
            return self.base + 4 * self.at[name]
        first = self.at[over] + self.sizes[over] - 1 if end else self.at[over] - self.sizes[name] + 1
        assert 0 <= first and first + self.sizes[name] <= self.all.numel()
        return self.base + 4 * first


def refused(memory, call, inputs, outputs, allowed):
    before = memory.all.clone()
    for out in outputs:
        for other in inputs + outputs:
            if other == out:
                continue
            for end in (False, True):
                with pytest.raises(tdp.TdpError) as e:
                    call({**{n: memory.ptr(n) for n in inputs + outputs}, out: memory.ptr(out, other, end)})
                assert e.value.code == tdp.EINVAL, (out, other, end)
            if (out, other) not in allowed:
                with pytest.raises(tdp.TdpError) as e:
                    call({**{n: memory.ptr(n) for n in inputs + outputs}, out: memory.ptr(other)})
                assert e.value.code == tdp.EINVAL, (out, other)
    torch.cuda.synchronize()
    assert torch.equal(before, memory.all)


# (a margin on both sides: an overlap may begin in front of the first array and end behind the last)
def test_fork():
    m = Memory(low=64, parents=4, add=4, src_tables=16, src_lens=4, refs_in=16, refs_out=16, dst_tables=16, dst_lens=4, copies=8, status=4, high=64)
    h = tdp.tdp_pages_create(tdp.PagesConfig(16, 4, 4))
    names = ["parents", "add", "src_tables", "src_lens", "refs_in"], ["refs_out", "dst_tables", "dst_lens", "copies", "status"]

    def call(a):
        tdp.tdp_pages_fork(h, a["parents"], a["src_tables"], a["src_lens"], 4, a["add"], 0, 4, a["refs_in"], a["refs_out"], a["dst_tables"], a["dst_lens"],
                           a["copies"], a["status"])
    refused(m, call, *names, {("refs_out", "refs_in")})
    call({**{n: m.ptr(n) for n in names[0] + names[1]}, "refs_out": m.ptr("refs_in")})
    # what a call does not use does not matter: no rows on either side, no parents, no lengths of their own
    status = i32([9] * 4)
    tdp.tdp_pages_fork(h, None, None, None, 0, None, 1, 0, m.ptr("refs_in"), m.ptr("refs_in"), m.ptr("refs_in"), m.ptr("refs_in"), m.ptr("refs_in"), status)
    torch.cuda.synchronize()
    assert status.tolist() == [0, 0, 0, 16]
    tdp.tdp_pages_destroy(h)


def test_compact():
    m = Memory(low=64, src_tables=16, lens=4, refs_in=16, refs_out=16, dst_tables=16, moves=10, status=4, high=64)
    h = tdp.tdp_pages_create(tdp.PagesConfig(16, 4, 4))
    names = ["src_tables", "lens", "refs_in"], ["refs_out", "dst_tables", "moves", "status"]

    def call(a):
        tdp.tdp_pages_compact(h, a["src_tables"], a["lens"], 4, 5, a["refs_in"], a["refs_out"], a["dst_tables"], a["moves"], a["status"])
    refused(m, call, *names, {("refs_out", "refs_in"), ("dst_tables", "src_tables")})
    call({**{n: m.ptr(n) for n in names[0] + names[1]}, "refs_out": m.ptr("refs_in"), "dst_tables": m.ptr("src_tables")})
    torch.cuda.synchronize()
    tdp.tdp_pages_destroy(h)


def test_select():
    m = Memory(low=64, scores=8, parent=6, token=6, score=6, finished=6, high=64)
    h = tdp.tdp_beams_create(tdp.BeamsConfig(8, 3))
    logits, done = torch.zeros((8, 32), device="cuda"), i32([0, 1] * 4)

    def call(a):
        tdp.tdp_beams_select(h, logits, tdp.F32, 2, 4, 32, 32, a["scores"], done, 0, 3, a["parent"], a["token"], a["score"], a["finished"])
    refused(m, call, ["scores"], ["parent", "token", "score", "finished"], set())
    # flags that take their own place: as many results as beams
    flags = [torch.empty((2, 4), dtype=torch.int32, device="cuda") for _ in range(3)]
    score = torch.empty((2, 4), device="cuda")
    wide = tdp.tdp_beams_create(tdp.BeamsConfig(8, 4))
    results = []
    for into in (flags[2], done):
        tdp.tdp_beams_select(wide, logits, tdp.F32, 2, 4, 32, 32, m.ptr("scores"), done, 0, 4, flags[0], flags[1], score, into)
        torch.cuda.synchronize()
        results.append((flags[0].tolist(), flags[1].tolist(), score.tolist(), into.view(-1).tolist()))
    assert results[0] == results[1] and results[0][0] == [[1, 3, 0, 0], [5, 7, 4, 4]]
    tdp.tdp_beams_destroy(h)
    tdp.tdp_beams_destroy(wide)


def test_attend():
    shape = W.StageShape("attend", 1, 64, 4, 2, 64, 64)
    with Stage(tdp, shape, 4, 3, 0, 0, 2, load_weights=False) as st:
        rows = 3 * 4 * 64
        both = torch.zeros(4 * rows, dtype=torch.bfloat16, device="cuda")
        for off in (0, 8, rows - 8, 4, rows - 4, -8, -rows + 8):
            with pytest.raises(tdp.TdpError) as e:
                tdp.tdp_stage_attend(st.h, 0, both[rows:], i32([1, 1, 1]), i32([[0, 1]] * 3), 3, None, 0, both[rows + off:])
            assert e.value.code == tdp.EINVAL, off
        for off in (rows, -rows):
            tdp.tdp_stage_attend(st.h, 0, both[rows:], i32([1, 1, 1]), i32([[0, 1]] * 3), 3, None, 0, both[rows + off:])
        torch.cuda.synchronize()
