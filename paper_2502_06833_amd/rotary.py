"""Norms of queries and keys for each head with the position rotation in the same pass (`ead_rotate` of include/ead.h).

    rotary = Rotary(128, 1e6, q_gain=w["q_norm"], k_gain=w["k_norm"])     # once per layer
    q, k = rotary(q, k, positions)                                       # from rows to rows
    q = cache.append(q, k, v, batch, rotary)                             # the same on the way to a paged cache
"""
from __future__ import annotations

import ctypes as C

from .binding import lib
from .paged import FP8, Rows, _check, _code, _current_device, _empty_like, _outputs, _positions, _rows, _stream_ptr


class RotaryDesc(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rotary_dim", C.c_int32), ("interleaved", C.c_int32), ("gain_per_head", C.c_int32), ("eps", C.c_float),
                ("inv_freq", C.c_void_p), ("q_gain", C.c_void_p), ("k_gain", C.c_void_p)]


class Rotary:
    """What a layer does to its queries and keys before attention.

    theta: pair i turns by position * theta^(-2 i / rotary_dim); inv_freq: or by position * inv_freq[i] (a tensor of rotary_dim / 2 numbers, for scaled
    positions).  rotary_dim: the first elements that are turned (a multiple of 16; all of head_dim if not said, 0: none).  interleaved: pairs are
    neighbours instead of i and i + rotary_dim / 2.  q_gain, k_gain: float32 [head_dim], or [heads, head_dim] both; a vector is
    x / sqrt(mean(x^2) + eps) * gain before it is turned.  Without a gain it is not normalised."""

    def __init__(self, head_dim, theta=1e4, *, rotary_dim=None, interleaved=False, inv_freq=None, q_gain=None, k_gain=None, eps=1e-6, device=None):
        import torch
        if head_dim not in (32, 64, 128):
            raise ValueError(f"head_dim {head_dim} is not one of 32, 64, 128")
        rotary_dim = head_dim if rotary_dim is None else rotary_dim
        if rotary_dim < 0 or rotary_dim > head_dim or rotary_dim % 16:
            raise ValueError(f"rotary_dim {rotary_dim} is no multiple of 16 from 0 to {head_dim}")
        gains = [g for g in (q_gain, k_gain) if g is not None]
        for g in gains:
            if not g.is_cuda or g.dtype != torch.float32 or g.dim() not in (1, 2) or g.shape[-1] != head_dim or not g.is_contiguous() or g.dim() != gains[0].dim() \
                    or g.get_device() != gains[0].get_device():
                raise ValueError(f"q_gain, k_gain: contiguous float32 [{head_dim}] or [heads, {head_dim}] on one GPU are needed")
        if device is None:
            device = gains[0].device if gains else "cuda"
        if inv_freq is None:
            if not theta > 0:
                raise ValueError(f"theta {theta} is not positive")
            inv_freq = float(theta) ** (-torch.arange(0, rotary_dim, 2, dtype=torch.float64) / max(rotary_dim, 1))
        elif inv_freq.dim() != 1 or inv_freq.shape[0] != rotary_dim // 2:
            raise ValueError(f"inv_freq: {rotary_dim // 2} numbers are needed")
        self.inv_freq = inv_freq.to(device=device, dtype=torch.float64).contiguous()
        if not self.inv_freq.is_cuda:
            raise ValueError("a Rotary's numbers lie on a GPU")
        self.q_gain, self.k_gain, self.head_dim, self._device = q_gain, k_gain, head_dim, self.inv_freq.get_device()
        if gains and gains[0].get_device() != self._device:
            raise ValueError("inv_freq and gains have to be on one GPU")
        self._heads = [g.shape[0] if g is not None and g.dim() == 2 else None for g in (q_gain, k_gain)]
        ptr = [g.data_ptr() if g is not None else None for g in (q_gain, k_gain)]
        self._desc = RotaryDesc(head_dim, rotary_dim, interleaved, bool(gains) and gains[0].dim() == 2, eps, self.inv_freq.data_ptr() if rotary_dim else None, *ptr)
        self._ref = C.byref(self._desc)
        self._rotate = lib().ead_rotate

    def _fits(self, head_dim, device, n_heads, n_kv_heads):
        if head_dim != self.head_dim or device != self._device:
            raise ValueError(f"vectors of {head_dim} on GPU {device}, but a Rotary for {self.head_dim} on GPU {self._device}")
        if self._desc.gain_per_head:
            for name, have, need in (("q_gain", self._heads[0], n_heads), ("k_gain", self._heads[1], n_kv_heads)):
                if have is not None and have != need:
                    raise ValueError(f"{name}: gains of {have} heads, {need} are needed")

    def __call__(self, q, k, positions, out=None):
        """(q, k) [rows, heads, head_dim] of float32 or bfloat16 (any row and head strides) normalised and turned by positions, int32 [rows]: new tensors, or
        `out` (which may be (q, k))."""
        if q.dim() != 3 or k.dim() != 3:
            raise ValueError(f"q, k: expected [rows, heads, {self.head_dim}], got {list(q.shape)} and {list(k.shape)}")
        code = _code(q)
        if code == FP8 or k.dtype != q.dtype:
            raise ValueError(f"q and k of one type, float32 or bfloat16, are needed, got {q.dtype} and {k.dtype}")
        rows, n_heads, n_kv = q.shape[0], q.shape[1], k.shape[1]
        self._fits(self.head_dim, self._device, n_heads, n_kv)
        rq, rk = _rows("q", q, self, rows, n_heads), _rows("k", k, self, rows, n_kv)
        if out is None:
            out = (_empty_like(q), _empty_like(k))
            dim = self.head_dim
            oq, ok = Rows(out[0].data_ptr(), n_heads * dim, dim), Rows(out[1].data_ptr(), n_kv * dim, dim)
        elif out[0].dtype != q.dtype or out[1].dtype != q.dtype:
            raise ValueError(f"out: {q.dtype} is needed, got {out[0].dtype} and {out[1].dtype}")
        else:
            oq, ok = _outputs("out", out[0], self, rows, n_heads), _outputs("out", out[1], self, rows, n_kv)
        at = _positions(positions, rows, self._device)
        stream = _stream_ptr()
        if _current_device() != self._device:
            raise ValueError(f"tensors on GPU {self._device}, but GPU {_current_device()} is the current one (torch.cuda.set_device, torch.cuda.device)")
        if rows and n_heads + n_kv:
            byref = C.byref
            rc = self._rotate(self._ref, code, rows, n_heads, n_kv, at, byref(rq), byref(rk), byref(oq), byref(ok), stream)
            if rc:
                _check(rc)
        return out
