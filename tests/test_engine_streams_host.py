"""Without a GPU: on which stream the worker's copies are.  torch's streams are replaced by names and device tensors by host ones; the
stage library's calls are recorded instead of made."""
import contextlib

import pytest
import torch

from paper_2506_10470_amd.engine import StageWorker


class Recorder:
    """The entry points that the worker calls, as (name, stream) pairs"""
    MAX_TOP = 32

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args[-1]))


@pytest.fixture
def streams(monkeypatch):
    class Stream:
        def __init__(self, name):
            self.name = name

        def wait_stream(self, other):
            State.waits.append((self.name, other.name, len(State.copies)))

    class State:
        kind, current, copies, waits = Stream, Stream("caller's"), [], []

    @contextlib.contextmanager
    def stream(s):
        before, State.current = State.current, s
        yield
        State.current = before

    def copied(self):
        State.copies.append(State.current.name)
        return self

    empty = torch.empty

    def empty_on_host(*args, device=None, **kw):
        State.copies.append(State.current.name)
        return empty(*args, **kw).zero_()

    monkeypatch.setattr(State, "copies", [])
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: State.current)
    monkeypatch.setattr(torch.Tensor, "cuda", copied)
    monkeypatch.setattr(torch.Tensor, "cpu", copied)
    monkeypatch.setattr(torch, "empty", empty_on_host)
    return State


@pytest.mark.parametrize("logprobs", [None, 0, 2])
@pytest.mark.parametrize("own", [True, False])
def test_copies_and_buffers_are_on_the_stream_of_the_calls(streams, own, logprobs):
    tdp, mine = Recorder(), streams.kind("worker's") if own else streams.current
    w = StageWorker(tdp, [1, 2], 3, 64, 8, 4, 4, 16, 4, [[5, 6, 7], [8]], stream=mine if own else None, check_tables=True, logprobs=logprobs)
    streams.current = streams.kind("another")       # the caller goes on elsewhere
    w.prefill([0, 1], [3, 1])
    w.decode(0, [0, 1], [3, 1])
    w.release([0, 1], 0)
    assert [len(g) for g in w.generated] == [2, 2] and streams.current.name == "another"
    assert tdp.calls and all(s is mine for _, s in tdp.calls)
    assert len(streams.copies) >= 8 and set(streams.copies) == {mine.name}
    # each event is behind what the caller's stream holds: prefill and decode wait in front of their first copy
    events = [(a, b) for a, b, _ in streams.waits]
    assert events == [(mine.name, "caller's")] * own + [(mine.name, "another")] * 2
    assert all(at < len(streams.copies) for _, _, at in streams.waits) and len({at for _, _, at in streams.waits}) == len(events)
