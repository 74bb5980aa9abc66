"""A paged K/V cache in the caller's tensors, and attention over it (the `ead_paged_*` calls of include/ead.h).

    cache = PagedCache.empty(n_pages, page_size, n_kv_heads, head_dim, torch.float8_e4m3fn)    # one per layer
    batch = PagedBatch.of(page_table, q_lens, kv_lens)                                         # one per step, for all layers
    cache.write(k, v, batch)                        # the new tokens' keys and values
    out = cache.attention(q, batch, window=4096, sinks=4)

`kv_lens` count the new tokens: sequence b's rows are the last `q_lens[b]` of its `kv_lens[b]` positions.
"""
from __future__ import annotations

import ctypes as C

from .binding import BF16, F32, EadError, _stream_ptr, lib

FP8 = 2


class CacheDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_pages", C.c_int32), ("page_size", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p)]


class BatchDesc(C.Structure):
    _fields_ = [("batch", C.c_int32), ("rows", C.c_int32), ("max_q", C.c_int32), ("min_q", C.c_int32), ("max_kv", C.c_int32),
                ("table_stride", C.c_int32), ("table_width", C.c_int32), ("page_table", C.c_void_p), ("q_starts", C.c_void_p),
                ("kv_lens", C.c_void_p)]


class Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64)]


class AttnDesc(C.Structure):
    _fields_ = [("n_heads", C.c_int32), ("dtype", C.c_int32), ("window", C.c_int32), ("sinks", C.c_int32), ("scale", C.c_float),
                ("one_term", C.c_int32)]


def _check(rc):
    if rc:
        raise EadError(rc, (lib().ead_last_error(None) or b"").decode())


def _fits(**numbers):
    """The descriptors hold 32 bits, to which ctypes cuts a number without a word."""
    for name, n in numbers.items():
        if not -2 ** 31 <= n < 2 ** 31:
            raise ValueError(f"{name}: {n} does not fit 32 bits")


def _codes():
    import torch
    return {torch.float32: F32, torch.bfloat16: BF16, torch.float8_e4m3fn: FP8}


_dtypes = None


def _code(t) -> int:
    global _dtypes
    if _dtypes is None:
        _dtypes = _codes()
    c = _dtypes.get(t.dtype)
    if c is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return c


def _rows(name, t, cache, rows, heads) -> Rows:
    dim = cache.head_dim
    shape = t.shape
    if len(shape) != 3 or shape[0] != rows or shape[1] != heads or shape[2] != dim:
        raise ValueError(f"{name}: expected [{rows}, {heads}, {dim}], got {list(shape)}")
    s = t.stride()
    if s[2] != 1 or t.get_device() != cache._device:
        raise ValueError(f"{name}: a tensor on the cache's GPU whose last dimension is contiguous is needed")
    return Rows(t.data_ptr(), s[0], s[1])


def _outputs(name, t, cache, rows, heads) -> Rows:
    """The same for a tensor that is written: every vector needs a place of its own."""
    r = _rows(name, t, cache, rows, heads)
    if (rows > 1 and r.row_stride < cache.head_dim) or (heads > 1 and r.head_stride < cache.head_dim):
        raise ValueError(f"{name}: vectors that overlap (strides {t.stride()}) cannot be written")
    return r


def _current_device():
    """The current device's number (the accessor that returns it plainly, where this torch has it, looked up once)."""
    global _current_device
    import torch
    _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    return _current_device()


def _stream(cache, batch):
    """The current stream, for a call of the cache's device."""
    if batch._device != cache._device:
        raise ValueError(f"cache on GPU {cache._device}, batch on GPU {batch._device}: one is needed")
    stream = _stream_ptr()
    if _current_device() != cache._device:
        raise ValueError(f"cache on GPU {cache._device}, but GPU {_current_device()} is the current one (torch.cuda.set_device, torch.cuda.device)")
    return stream


def _empty_like(q):
    """A dense tensor of q's shape and type (torch.empty with a device takes three times as long on the host)."""
    import torch
    return torch.empty_like(q) if q.is_contiguous() else q.new_empty(q.shape)


def _empty_f32(q, *shape):
    import torch
    return q.new_empty(shape, dtype=torch.float32)


def _capturing():
    """Whether the current stream is being captured (torch's accessor, looked up once)."""
    global _capturing
    import torch
    _capturing = torch.cuda.is_current_stream_capturing
    return _capturing()


class PagedBatch:
    """What a step works on.  page_table [batch, width] (rows of its own for every sequence, not an expanded one), q_starts [batch + 1]
    and kv_lens [batch] are int32 tensors on the GPU and stay the caller's: they may be changed in place between calls as long as the
    bounds hold.

    A batch keeps the workspaces of `PagedCache.attention`, one for each stream.  Calls under a graph capture get one that belongs to the
    graph: it lies in the graph's memory and a node of the graph clears it, so captures need no call before them, and graphs of one batch
    may run beside each other and beside eager calls."""

    def __init__(self, page_table, q_starts, kv_lens, *, rows, max_q, max_kv, min_q=0):
        import torch
        for name, t, dims in (("page_table", page_table, 2), ("q_starts", q_starts, 1), ("kv_lens", kv_lens, 1)):
            if not t.is_cuda or t.dtype != torch.int32 or t.dim() != dims or t.stride(-1) != 1:
                raise ValueError(f"{name}: an int32 tensor on the GPU with {dims} dimension(s), the last contiguous, is needed")
        n = page_table.shape[0]
        if q_starts.shape[0] != n + 1 or kv_lens.shape[0] != n:
            raise ValueError(f"{n} sequences in page_table need q_starts of {n + 1} and kv_lens of {n}")
        if page_table.device != q_starts.device or page_table.device != kv_lens.device:
            raise ValueError("page_table, q_starts and kv_lens have to be on one device")
        width = page_table.shape[1]
        stride = page_table.stride(0) if n > 1 else width         # a single row's stride says nothing
        if stride < width:
            raise ValueError("page_table: its rows overlap (an expanded table?); .contiguous() gives every sequence its own")
        _fits(rows=rows, max_q=max_q, min_q=min_q, max_kv=max_kv, stride=stride)
        self.page_table, self.q_starts, self.kv_lens = page_table, q_starts, kv_lens
        self.rows = rows
        self._device = page_table.get_device()
        self._desc = BatchDesc(n, rows, max_q, min_q, max_kv, stride, width, page_table.data_ptr(), q_starts.data_ptr(), kv_lens.data_ptr())
        self._ref = C.byref(self._desc)
        self._plans = {}
        self._of_capture = (None, {})

    @classmethod
    def of(cls, page_table, q_lens, kv_lens):
        """From host lengths; page_table may be a GPU tensor or rows of page numbers (of any lengths)."""
        import torch
        if not hasattr(page_table, "is_cuda"):
            width = max([len(r) for r in page_table] + [1])
            page_table = torch.tensor([list(r) + [-1] * (width - len(r)) for r in page_table], dtype=torch.int32).cuda()
        q_lens, kv_lens = [int(n) for n in q_lens], [int(n) for n in kv_lens]
        if len(q_lens) != len(kv_lens) or min(q_lens + kv_lens, default=0) < 0:
            raise ValueError("q_lens and kv_lens: one length of 0 or more for each sequence")
        starts = [0]
        for n in q_lens:
            starts.append(starts[-1] + n)
        dev = page_table.device
        return cls(page_table, torch.tensor(starts, dtype=torch.int32).to(dev), torch.tensor(kv_lens, dtype=torch.int32).to(dev),
                   rows=starts[-1], max_q=max(q_lens, default=0), min_q=min(q_lens, default=0), max_kv=max(kv_lens, default=0))

    def _captured_plans(self, stream):
        """The plans of the capture under way: they go with the next one, and their memory is the graph's until then and after."""
        n = C.c_uint64(0)
        _check(lib().ead_stream_capture(C.c_void_p(stream), C.byref(n)))
        if self._of_capture[0] != n.value:
            self._of_capture = (n.value, {})
        return self._of_capture[1]

    def _plan(self, cache, n_heads, window, sinks, scale, one_term, stream):
        """The attention arguments, and the workspace of this stream: cleared once, then every call leaves it ready for the next."""
        plans = self._captured_plans(stream) if _capturing() else self._plans
        key = (stream, cache._key, n_heads, window, sinks, scale, one_term)
        p = plans.get(key)
        if p is None:
            import torch
            _fits(window=window, sinks=sinks)
            d = AttnDesc(n_heads, F32 if cache._code == F32 else BF16, window, sinks, scale, one_term)
            need = C.c_uint64(0)
            _check(lib().ead_paged_workspace(cache._ref, self._ref, C.byref(d), C.byref(need)))
            ws = torch.zeros((need.value + 3) // 4, dtype=torch.int32, device=self.kv_lens.device) if need.value else None
            p = plans[key] = (C.byref(d), ws.data_ptr() if need.value else None, need.value, d, ws)
        return p


class PagedCache:
    """The cache of one attention layer: k_pages, v_pages [n_pages, n_kv_heads, page_size, head_dim] in float32, bfloat16 or
    float8_e4m3fn, the last with k_scales, v_scales [n_pages, n_kv_heads, page_size] uint8 (a vector is its codes times
    2^(scale - 127)).  The tensors are the caller's."""

    def __init__(self, k_pages, v_pages, k_scales=None, v_scales=None):
        import torch
        if k_pages.dim() != 4 or k_pages.shape != v_pages.shape or k_pages.dtype != v_pages.dtype:
            raise ValueError("k_pages and v_pages: two [n_pages, n_kv_heads, page_size, head_dim] of one type are needed")
        self._code = _code(k_pages)
        scales = () if self._code != FP8 else (k_scales, v_scales)
        if (self._code == FP8) != (k_scales is not None) or (k_scales is None) != (v_scales is None):
            raise ValueError("k_scales and v_scales go with float8_e4m3fn pages, and with no others")
        for t in (k_pages, v_pages) + scales:
            if not t.is_cuda or not t.is_contiguous() or t.device != k_pages.device:
                raise ValueError("pages and scales have to be contiguous and on one GPU")
        for t in scales:
            if t.dtype != torch.uint8 or t.shape != k_pages.shape[:3]:
                raise ValueError("scales: uint8 [n_pages, n_kv_heads, page_size] are needed")
        self.k_pages, self.v_pages, self.k_scales, self.v_scales = k_pages, v_pages, k_scales, v_scales
        n, self.n_kv_heads, self.page_size, self.head_dim = k_pages.shape
        ptr = [t.data_ptr() if t is not None else None for t in (k_pages, v_pages, k_scales, v_scales)]
        self._desc = CacheDesc(self._code, n, self.page_size, self.n_kv_heads, self.head_dim, *ptr)
        self._ref = C.byref(self._desc)
        _fits(n_pages=n)
        self._device = k_pages.get_device()
        self._key = (self._code, self.page_size, self.n_kv_heads, self.head_dim)
        self._attention = lib().ead_paged_attention
        self._scale = 1.0 / float(self.head_dim) ** 0.5

    @classmethod
    def empty(cls, n_pages, page_size, n_kv_heads, head_dim, dtype, device="cuda"):
        """Pages that hold nothing yet (their memory is not cleared: what no position has been written to is never used)."""
        import torch
        pages = [torch.empty((n_pages, n_kv_heads, page_size, head_dim), dtype=dtype, device=device) for _ in range(2)]
        if dtype == torch.float8_e4m3fn:
            pages += [torch.empty((n_pages, n_kv_heads, page_size), dtype=torch.uint8, device=device) for _ in range(2)]
        return cls(*pages)

    def write(self, k, v, batch):
        """Keys and values [rows, n_kv_heads, head_dim] (float32 or bfloat16, any row and head strides) of the batch's rows."""
        code = _code(k)
        if v.dtype != k.dtype:
            raise ValueError(f"k and v of one type are needed, got {k.dtype} and {v.dtype}")
        rk = _rows("k", k, self, batch.rows, self.n_kv_heads)
        rv = _rows("v", v, self, batch.rows, self.n_kv_heads)
        stream = _stream(self, batch)
        if batch.rows:
            _check(lib().ead_paged_write(self._ref, batch._ref, code, C.byref(rk), C.byref(rv), stream))

    def read(self, batch, dtype=None, out=None):
        """(k, v) [rows, n_kv_heads, head_dim] of the batch's rows, as `dtype` (bfloat16 if not said) or into `out`."""
        import torch
        if out is None:
            k = self.k_pages.new_empty((batch.rows, self.n_kv_heads, self.head_dim), dtype=torch.bfloat16 if dtype is None else dtype)
            out = (k, torch.empty_like(k))
        k, v = out
        if v.dtype != k.dtype:
            raise ValueError(f"out of one type is needed, got {k.dtype} and {v.dtype}")
        rk = _outputs("k", k, self, batch.rows, self.n_kv_heads)
        rv = _outputs("v", v, self, batch.rows, self.n_kv_heads)
        stream = _stream(self, batch)
        if batch.rows:
            _check(lib().ead_paged_read(self._ref, batch._ref, _code(k), C.byref(rk), C.byref(rv), stream))
        return out

    def attention(self, q, batch, window=0, sinks=0, scale=None, want_lse=False, out=None, one_term=False):
        """softmax(scale q K^T) V of the batch's rows over their sequences, [rows, n_heads, head_dim] of q's type: float32
        over a float32 cache, bfloat16 over the others.  A row sees the positions up to its own; with window > 0 the last
        `window` of them and the first `sinks` of the sequence.  scale: 1 / sqrt(head_dim) if not said.  want_lse: also the
        logarithm of the sum of exponentials, [rows, n_heads] float32.  Rows that see nothing get 0 and -inf.  one_term:
        prompts' rows over 16- and 8-bit pages may take their probabilities with 8 bits instead of 16, for a quarter less time over
        thousands of keys (error against 64 bits 0.0023 of the output's norm instead of 0.0017)."""
        if q.dim() != 3:
            raise ValueError(f"q: expected [rows, n_heads, {self.head_dim}], got {list(q.shape)}")
        if _code(q) != (F32 if self._code == F32 else BF16):
            raise ValueError(f"{q.dtype} queries over {self.k_pages.dtype} pages: float32 over float32, bfloat16 over the others")
        rows, n_heads = batch.rows, q.shape[1]
        rq = _rows("q", q, self, rows, n_heads)
        if out is None:
            out = _empty_like(q)
        elif out.dtype != q.dtype:
            raise ValueError(f"out: {q.dtype} is needed, got {out.dtype}")
        ro = _outputs("out", out, self, rows, n_heads)
        lse = _empty_f32(q, rows, n_heads) if want_lse else None
        stream = _stream(self, batch)
        p = batch._plan(self, n_heads, window, sinks, self._scale if scale is None else scale, one_term, stream)
        rc = self._attention(self._ref, batch._ref, p[0], C.byref(rq), C.byref(ro), lse.data_ptr() if want_lse else None, p[1], p[2], stream)
        if rc:
            _check(rc)
        return (out, lse) if want_lse else out
