"""Two threads' calls of logprobs on one stream, without a GPU: another thread may get in between a call's look at its workspace and its launch."""
import ctypes as C
import gc
import weakref

import pytest
import torch

from paper_2502_06833_amd import paged, scoring
from test_paged_arguments import OnGpu


class Library:
    """The calls that logprobs makes; `meanwhile` runs inside the first launch, where the interpreter lets other threads in."""

    def __init__(self, meanwhile):
        self.meanwhile, self.seen = meanwhile, []

    def ead_logprobs_workspace(self, ref, n):
        C.cast(n, C.POINTER(C.c_uint64))[0] = 4096 * ref._obj.rows
        return 0

    def ead_stream_capture(self, stream, n):
        C.cast(n, C.POINTER(C.c_uint64))[0] = stream.value or 0
        return 0

    def ead_logprobs(self, ref, workspace, size, stream):
        run, self.meanwhile = self.meanwhile, None
        if run:
            run()
        self.seen.append((ref._obj.rows, workspace, size))
        return 0


@pytest.fixture
def made(monkeypatch):
    """Workspaces in host memory: (address, bytes, whether it still exists)."""
    made, zeros = [], torch.zeros

    def host_zeros(*shape, device=None, **kw):
        t = zeros(*shape, **kw)
        made.append((t.data_ptr(), t.numel() * 4, weakref.ref(t)))
        return t

    monkeypatch.setattr(torch, "zeros", host_zeros)
    monkeypatch.setattr(scoring, "_workspaces", scoring._Workspaces())
    monkeypatch.setattr(scoring, "_needs", {})
    monkeypatch.setattr(scoring, "_stream_ptr", lambda: 7)
    monkeypatch.setattr(paged, "_current_device", lambda: 0)
    monkeypatch.setattr(paged, "_capturing", lambda: False)
    return made


def logits(rows):
    return OnGpu(torch.empty(rows, 64, dtype=torch.float32))


@pytest.mark.parametrize("capturing", [False, True])
@pytest.mark.parametrize("first,second", [(2, 9), (9, 2), (3, 3)])
def test_a_workspace_lives_until_its_launch(made, monkeypatch, capturing, first, second):
    """The second call replaces the first one's workspace if it needs more: the first's memory has to be there when its kernel is launched."""
    monkeypatch.setattr(paged, "_capturing", lambda: capturing)
    held = []

    def meanwhile():
        scoring.logprobs(logits(second))
        gc.collect()
        held.append([alive() is not None for at, _, alive in made if at == mine[0]])

    L = Library(meanwhile)
    monkeypatch.setattr(scoring, "lib", lambda: L)
    monkeypatch.setattr(paged, "lib", lambda: L)
    launch, mine = L.ead_logprobs, []

    def first_sees(ref, workspace, size, stream):
        mine.append(workspace)
        return launch(ref, workspace, size, stream)

    L.ead_logprobs = first_sees
    scoring.logprobs(logits(first))
    assert held == [[True]]
    assert sorted(rows for rows, _, _ in L.seen) == sorted((first, second))
    for rows, at, size in L.seen:                             # every launch got as much as it asked for
        assert size == 4096 * rows and any(at == a and n >= size for a, n, _ in made)


def test_captures_of_two_threads_do_not_mix(made, monkeypatch):
    """A second capture that begins between a call's look at the captures and its workspace's place among them: none gets the other's memory."""
    w = scoring._workspaces
    monkeypatch.setattr(paged, "_capturing", lambda: True)
    L = Library(None)
    monkeypatch.setattr(scoring, "lib", lambda: L)

    class Slot(tuple):
        """A capture's workspaces whose first look lets another thread's capture in."""

        def __getitem__(self, i):
            if Slot.meanwhile:
                run, Slot.meanwhile = Slot.meanwhile, None
                run()
            return tuple.__getitem__(self, i)

    w.get(64, 0, 1)
    w._captured = Slot(w._captured)
    Slot.meanwhile = lambda: w.get(64, 0, 2)
    w.get(64, 0, 1)
    assert w._captured[0] == (0, 2) and set(w._captured[1]) == {(0, 2)}
