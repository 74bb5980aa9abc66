"""Captures of two threads at once over one batch, without a GPU."""
import ctypes as C

import torch

from paper_2502_06833_amd import paged
from test_paged_arguments import batch_of


class Library:
    def ead_stream_capture(self, stream, n):
        C.cast(n, C.POINTER(C.c_uint64))[0] = stream.value
        return 0


def test_captures_of_two_threads_do_not_mix(monkeypatch):
    """A second capture that begins between a call's look at the batch's capture and at its plans: the first gets its own plans, not the second's."""
    monkeypatch.setattr(paged, "lib", lambda: Library())
    b = batch_of(torch.zeros(2, 3, dtype=torch.int32))
    first = b._captured_plans(1)

    class Slot(tuple):
        def __getitem__(self, i):
            if Slot.meanwhile:
                run, Slot.meanwhile = Slot.meanwhile, None
                run()
            return tuple.__getitem__(self, i)

    b._of_capture, theirs = Slot(b._of_capture), []
    Slot.meanwhile = lambda: theirs.append(b._captured_plans(2))
    assert b._captured_plans(1) is first and theirs[0] is not first
    assert b._captured_plans(2) is theirs[0]
