"""Log probabilities of given tokens, entropies and the most likely tokens from logits (`ead_logprobs` of include/ead.h)."""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple

from .binding import BF16, F32, NATS, _stream_ptr, lib
from . import paged
from .paged import _check


class CallDesc(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("dtype", C.c_int32), ("rows", C.c_int32), ("vocab", C.c_int32), ("row_stride", C.c_int64), ("tokens", C.c_void_p),
                ("top", C.c_int32), ("unit", C.c_int32), ("logprob", C.c_void_p), ("H", C.c_void_p), ("rank", C.c_void_p), ("top_tokens", C.c_void_p),
                ("top_logprobs", C.c_void_p)]


class LogProbs(NamedTuple):
    H: object                   # [rows] float32: entropies
    logprob: object = None      # [rows] float32: of the given tokens (0 where there is none)
    rank: object = None         # [rows] int32: 1 + the number of larger logits (0 where there is no token)
    top_tokens: object = None   # [rows, top] int32: the most likely tokens, equal ones in their order
    top_logprobs: object = None  # [rows, top] float32


class _Workspaces:
    """One for each stream, cleared when it is made; calls leave it ready for the next.  A capture's calls have one for each of its streams, in the graph's memory and
    cleared by a node of the graph.  Threads share them: a call holds the tensor that it got until its kernel is launched, since another thread's call on the same
    stream may meanwhile put a larger one in its place (after that the stream's order keeps them apart)."""

    def __init__(self):
        self._eager, self._captured = {}, (None, {})

    def get(self, need, device, stream):
        of, key = self._eager, (device, stream)
        if paged._capturing():
            n = C.c_uint64(0)
            _check(lib().ead_stream_capture(C.c_void_p(stream), C.byref(n)))
            captured = self._captured                          # (read once: another thread's capture may replace it)
            if captured[0] != (device, n.value):
                captured = self._captured = ((device, n.value), {})
            of = captured[1]
        ws = of.get(key)
        if ws is None or ws.numel() * 4 < need:
            import torch
            ws = of[key] = torch.zeros((need + 3) // 4, dtype=torch.int32, device=torch.device("cuda", device))
        return ws


_workspaces = _Workspaces()
_dtypes = None
_needs = {}                     # (rows, vocab, top): bytes


def logprobs(logits, tokens=None, top=0, unit=NATS):
    """logits [rows, vocab], bfloat16 or float32, any row stride; tokens: int32 [rows] (outside 0 .. vocab-1: none); top: alternatives, 0 .. 32.
    Log probabilities are natural logarithms, entropies in `unit`.  Rows without a distribution (a NaN, +inf, nothing above -inf) have NaN."""
    import torch
    global _dtypes
    if _dtypes is None:
        _dtypes = {torch.float32: F32, torch.bfloat16: BF16}
    code = _dtypes.get(logits.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {logits.dtype}")
    if not logits.is_cuda or logits.dim() != 2:
        raise ValueError("logits: [rows, vocab] on the GPU are needed")
    (rows, vocab), (stride, apart) = logits.shape, logits.stride()
    if apart != 1 and vocab > 1:
        raise ValueError("logits: rows whose elements lie side by side are needed")
    if vocab < 1 or top < 0 or top > min(32, vocab):
        raise ValueError(f"top {top} is not in 0 .. {min(32, vocab)} (vocab {vocab})")
    device = logits.get_device()
    if tokens is not None and (tokens.dtype != torch.int32 or tokens.shape != (rows,) or (rows > 1 and tokens.stride(0) != 1) or tokens.get_device() != device):
        raise ValueError(f"tokens: int32 [{rows}], contiguous and on the logits' GPU, is needed")
    if paged._current_device() != device:
        raise ValueError(f"logits on GPU {device}, but GPU {paged._current_device()} is the current one (torch.cuda.set_device, torch.cuda.device)")
    f32, i32 = torch.float32, torch.int32
    H = logits.new_empty(rows, dtype=f32)
    lp, rank = (logits.new_empty(rows, dtype=f32), logits.new_empty(rows, dtype=i32)) if tokens is not None else (None, None)
    tt, tl = (logits.new_empty((rows, top), dtype=i32), logits.new_empty((rows, top), dtype=f32)) if top else (None, None)
    given, more = tokens is not None, top > 0
    d = CallDesc(logits.data_ptr(), code, rows, vocab, stride if rows > 1 else vocab, tokens.data_ptr() if given else None, top, unit, lp.data_ptr() if given else None,
                 H.data_ptr(), rank.data_ptr() if given else None, tt.data_ptr() if more else None, tl.data_ptr() if more else None)
    ref, stream = C.byref(d), _stream_ptr()
    need = _needs.get((rows, vocab, top))
    if need is None:
        n = C.c_uint64(0)
        _check(lib().ead_logprobs_workspace(ref, C.byref(n)))
        if len(_needs) >= 1024:
            _needs.clear()
        need = _needs[rows, vocab, top] = n.value
    ws = _workspaces.get(need, device, stream) if need else None
    rc = lib().ead_logprobs(ref, ws.data_ptr() if need else None, need, stream)
    if rc:
        _check(rc)
    return LogProbs(H, lp, rank, tt, tl)
