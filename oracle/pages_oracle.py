"""Block tables that fork and compact, page by page in plain Python: what tdp_pages_fork and tdp_pages_compact are checked against."""
from __future__ import annotations

from typing import List, Optional, Sequence, Tuple

PAGE = 16


def pages_of(tokens: int) -> int:
    return -(-tokens // PAGE)


def fork(parents: Sequence[int], tables: Sequence[Sequence[int]], lens: Sequence[int], add: Sequence[int], refs: Sequence[int], width: int):
    """-> (tables, lens, refs, copies, status), tables and lens None where nothing happens."""
    n_src, most = len(lens), width * PAGE
    free = [p for p, n in enumerate(refs) if n == 0]
    bad = 0
    for p, a in zip(parents, add):
        n = lens[p] if 0 <= p < n_src else 0
        ok = -1 <= p < n_src and 0 <= n <= most and 0 <= a <= most - n
        if ok and n % PAGE:
            ok = 0 <= tables[p][n // PAGE] < len(refs)
        bad += not ok
    if not bad and any(not 0 <= n <= most for n in lens):
        bad = 1
    if bad:
        # (what is missing is counted over the rows that are in order)
        return None, None, list(refs), [(-1, -1)] * len(parents), bad
    new, copies, taken, seen = [], [], 0, set()
    wanted: List[List[Optional[int]]] = []
    for p, a in zip(parents, add):
        n = lens[p] if p >= 0 else 0
        row: List[Optional[int]] = list(tables[p][:pages_of(n)]) if p >= 0 else []
        copy = -1
        if n % PAGE:
            if not (p not in seen and refs[row[-1]] == 1):
                copy, row[-1] = row[-1], None
        seen.add(p)
        row += [None] * (pages_of(n + a) - len(row))
        taken += row.count(None)
        wanted.append(row)
        copies.append(copy)
    if taken > len(free):
        return None, None, list(refs), [(-1, -1)] * len(parents), (taken - len(free), 0, 0, len(free))
    out = list(refs)
    for row, n in zip(tables, lens):
        for p in row[:pages_of(n)]:
            out[p] -= 1
    it, pairs = iter(free), []
    for row, copy in zip(wanted, copies):
        fresh = None
        full: List[int] = []
        for p in row:
            if p is None:
                p = next(it)
                fresh = p if fresh is None else fresh
            full.append(p)
            out[p] += 1
        pairs.append((copy, fresh) if copy >= 0 else (-1, -1))
        new.append(full + [-1] * (width - len(full)))
    return new, [(lens[p] if p >= 0 else 0) + a for p, a in zip(parents, add)], out, pairs, (0, 0, taken, len(free))


def compact(tables: Sequence[Sequence[int]], lens: Sequence[int], refs: Sequence[int], max_moves: int, width: int):
    """-> (tables, refs, moves, status)"""
    named = [0] * len(refs)
    bad = 0
    for row, n in zip(tables, lens):
        ok = 0 <= n <= width * PAGE
        if ok:
            for p in row[:pages_of(n)]:
                if 0 <= p < len(refs):
                    named[p] += 1
                else:
                    ok = False
        bad += not ok
    free = [p for p, n in enumerate(refs) if n == 0]
    movable = [p for p in range(len(refs) - 1, -1, -1) if refs[p] > 0 and named[p] == refs[p]]
    used = sum(n > 0 for n in refs)
    moves: List[Tuple[int, int]] = []
    if not bad:
        for k in range(min(max_moves, len(free), len(movable))):
            if free[k] >= movable[k]:
                break
            moves.append((movable[k], free[k]))
    to, out = dict(moves), list(refs)
    for a, b in moves:
        out[b], out[a] = out[a], 0
    new = []
    for row, n in zip(tables, lens):
        held = pages_of(min(max(n, 0), width * PAGE))
        new.append([to.get(p, p) for p in row[:held]] + [-1] * (width - held))
    return new, out, moves + [(-1, -1)] * (max_moves - len(moves)), (0, bad, len(moves), used)
