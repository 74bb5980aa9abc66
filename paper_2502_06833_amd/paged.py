"""A paged K/V cache in the caller's tensors, and attention over it (the `ead_paged_*` calls of include/ead.h).

    cache = PagedCache.empty(n_pages, page_size, n_kv_heads, head_dim, torch.float8_e4m3fn)    # one per layer
    batch = PagedBatch.of(page_table, q_lens, kv_lens)                                         # one per step, for all layers
    cache.write(k, v, batch)                        # the new tokens' keys and values
    out = cache.attention(q, batch, window=4096, sinks=4)

and the steps around it (`Rotary` is in rotary.py):

    q = cache.append(q, k, v, batch, rotary)        # queries and keys normalised and rotated, keys and values written
    out, lse = cache.attention(q, batch, want_lse=True)
    cache.weigh(q, lse, batch, weights)             # what every position is paid, added up in weights = cache.new_weights()
    kept = cache.evict(batch, weights, 2048, sinks=4, recent=256)    # afterwards sequences hold kv_lens.clamp(max=2048) positions

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


class EvictionDesc(C.Structure):
    _fields_ = [("keep", C.c_int32), ("sinks", C.c_int32), ("recent", C.c_int32)]


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


def _cross(rows, heads, row, head, dim):
    """Whether two vectors of different rows and heads share an element: some multiple of one stride lies within `dim` of one of the other."""
    for h in range(1, heads):
        r = h * head // row
        if (r < rows and h * head - r * row < dim) or (r + 1 < rows and (r + 1) * row - h * head < dim):
            return True
    return False


def _outputs(name, t, cache, rows, heads) -> Rows:
    """The same for a tensor that is written: every vector needs a place of its own."""
    r = _rows(name, t, cache, rows, heads)
    row, head, dim = r.row_stride, r.head_stride, cache.head_dim
    if (rows > 1 and row < dim) or (heads > 1 and head < dim) or (rows > 1 and heads > 1 and row < (heads - 1) * head + dim and _cross(rows, heads, row, head, dim)):
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
        of = self._of_capture                                 # (read once: another thread's capture of the batch may replace it)
        if of[0] != n.value:
            of = self._of_capture = (n.value, {})
        return of[1]

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

    def _sized(self, what, cache, args, describe):
        """A call's descriptor and the bytes of the workspace it wants, which nothing has to clear."""
        key = (what, cache._key, args)
        p = self._plans.get(key)
        if p is None:
            d = describe(*args)
            need = C.c_uint64(0)
            _check(getattr(lib(), what)(cache._ref, self._ref, C.byref(d), C.byref(need)))
            p = self._plans[key] = (C.byref(d), need.value, d)
        return p


def _scratch(like, need):
    """Device memory for one call on the current stream (or in the graph that is being captured)."""
    import torch
    return like.new_empty((need + 3) // 4, dtype=torch.int32) if need else None


def _positions(t, rows, device):
    import torch
    if t.dtype != torch.int32 or t.dim() != 1 or t.shape[0] != rows or (rows > 1 and t.stride(0) != 1) or t.get_device() != device:
        raise ValueError(f"positions: int32 [{rows}], contiguous and on the same GPU, is needed")
    return t.data_ptr()


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
        self._attention, self._append, self._weigh = lib().ead_paged_attention, lib().ead_paged_append, lib().ead_paged_weigh
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

    def append(self, q, k, v, batch, rotary, positions=None, out=None):
        """The batch's queries [rows, n_heads, head_dim] normalised and turned (into `out`, or a new tensor; `out` may be q), its keys
        likewise and its values as they are written to their places, all in one pass.  q, k, v: float32 or bfloat16, any row and head strides.
        rotary: a Rotary.  positions: int32 [rows]; the batch's own if not said, which are a text's as long as nothing has been evicted."""
        if q.dim() != 3:
            raise ValueError(f"q: expected [rows, n_heads, {self.head_dim}], got {list(q.shape)}")
        code = _code(q)
        if code == FP8 or k.dtype != q.dtype or v.dtype != q.dtype:
            raise ValueError(f"q, k and v of one type, float32 or bfloat16, are needed, got {q.dtype}, {k.dtype} and {v.dtype}")
        rows, n_heads = batch.rows, q.shape[1]
        rotary._fits(self.head_dim, self._device, n_heads, self.n_kv_heads)
        rq = _rows("q", q, self, rows, n_heads)
        rk = _rows("k", k, self, rows, self.n_kv_heads)
        rv = _rows("v", v, self, rows, self.n_kv_heads)
        if out is None:
            out = _empty_like(q)
            ro = Rows(out.data_ptr(), n_heads * self.head_dim, self.head_dim)
        elif out.dtype != q.dtype:
            raise ValueError(f"out: {q.dtype} is needed, got {out.dtype}")
        else:
            ro = _outputs("out", out, self, rows, n_heads)
        at = None if positions is None else _positions(positions, rows, self._device)
        stream = _stream(self, batch)
        if rows:
            byref = C.byref
            rc = self._append(self._ref, batch._ref, rotary._ref, code, n_heads, at, byref(rq), byref(rk), byref(rv), byref(ro), stream)
            if rc:
                _check(rc)
        return out

    def new_weights(self):
        """Float32 pages for `weigh`, [n_pages, n_kv_heads, page_size], all zero."""
        import torch
        return torch.zeros(self.k_pages.shape[:3], dtype=torch.float32, device=self.k_pages.device)

    def _pool(self, name, t):
        import torch
        if t.dtype != torch.float32 or t.shape != self.k_pages.shape[:3] or not t.is_contiguous() or t.get_device() != self._device:
            raise ValueError(f"{name}: contiguous float32 {list(self.k_pages.shape[:3])} on the cache's GPU is needed")
        return t.data_ptr()

    def weigh(self, q, lse, batch, weights, window=0, sinks=0, scale=None):
        """Adds to `weights` (float32 [n_pages, n_kv_heads, page_size], see new_weights) what the rows' attention pays to every position
        they see, exp(scale q k - lse) over the rows and the query heads of a group; the rows' own positions start from nothing.  q, window, sinks and
        scale as for `attention` of the same rows, lse as it returned it.  A page belongs to one sequence of the batch; weights of positions
        that a window has passed are left alone (their pages may be others' by now), though their keys are still read."""
        if q.dim() != 3:
            raise ValueError(f"q: expected [rows, n_heads, {self.head_dim}], got {list(q.shape)}")
        if _code(q) != (F32 if self._code == F32 else BF16):
            raise ValueError(f"{q.dtype} queries over {self.k_pages.dtype} pages: float32 over float32, bfloat16 over the others")
        import torch
        rows, n_heads = batch.rows, q.shape[1]
        rq = _rows("q", q, self, rows, n_heads)
        if lse.dtype != torch.float32 or lse.shape != (rows, n_heads) or not lse.is_contiguous() or lse.get_device() != self._device:
            raise ValueError(f"lse: contiguous float32 [{rows}, {n_heads}] on the cache's GPU is needed")
        to = self._pool("weights", weights)
        stream = _stream(self, batch)
        _fits(window=window, sinks=sinks)
        args = (n_heads, F32 if self._code == F32 else BF16, window, sinks, self._scale if scale is None else scale, 0)
        d, need, _ = batch._sized("ead_paged_weigh_workspace", self, args, AttnDesc)
        ws = _scratch(lse, need)
        rc = self._weigh(self._ref, batch._ref, d, C.byref(rq), lse.data_ptr(), to, ws.data_ptr() if need else None, need, stream)
        if rc:
            _check(rc)
        return weights

    def evict(self, batch, scores, keep, sinks=0, recent=0, weights=None, kept=None):
        """Cuts every sequence of more than `keep` positions to that many, each KV head for itself: the first `sinks` and the last `recent`
        stay, and of the others those with the largest `scores` (float32 pages as those of `weigh`; of equal ones the lower positions).  The places
        that became free are filled from behind and the last positions follow, so the first `sinks` and the last `recent` keep
        their order.  `weights`: pages that move with the positions, `scores` if not said.  Returns int32 [sequences, n_kv_heads, keep]: which
        position lies where now (-1 past a sequence's end).  batch.kv_lens stays as it is, for the other layers; then it is
        kv_lens.clamp(max=keep)."""
        import torch
        _fits(keep=keep, sinks=sinks, recent=recent)
        if keep < 1 or sinks < 0 or recent < 0 or sinks + recent > keep:
            raise ValueError(f"keep {keep}, sinks {sinks}, recent {recent}: 1 or more, 0 or more, and sinks + recent <= keep are needed")
        n = batch._desc.batch
        of = self._pool("scores", scores)
        to = of if weights is None else self._pool("weights", weights)
        if kept is None:
            kept = scores.new_empty((n, self.n_kv_heads, keep), dtype=torch.int32)
        elif kept.dtype != torch.int32 or kept.shape != (n, self.n_kv_heads, keep) or not kept.is_contiguous() or kept.get_device() != self._device:
            raise ValueError(f"kept: contiguous int32 {[n, self.n_kv_heads, keep]} on the cache's GPU is needed")
        stream = _stream(self, batch)
        if n == 0:
            return kept
        d, need, _ = batch._sized("ead_paged_evict_workspace", self, (keep, sinks, recent), EvictionDesc)
        ws = _scratch(scores, need)
        _check(lib().ead_paged_evict(self._ref, batch._ref, d, of, to, kept.data_ptr(), ws.data_ptr(), need, stream))
        return kept
