"""What PagedBatch and PagedCache make of their tensors, without a GPU: stand-ins say that they lie on one."""
import ctypes as C
import threading

import pytest
import torch

import paper_2502_06833_amd as ead
from paper_2502_06833_amd import paged


class OnGpu:
    """A CPU tensor that says it is on a GPU: for checks and descriptors, which never touch the data."""

    def __init__(self, t, device="cuda:0"):
        self.t, self.device, self.is_cuda = t, torch.device(device), True

    def get_device(self):
        return self.device.index

    def __getattr__(self, name):
        return getattr(self.t, name)


def batch_of(page_table, device="cuda:0", **kw):
    n = page_table.shape[0]
    lens = torch.zeros(n, dtype=torch.int32)
    bounds = dict(rows=n, max_q=1, max_kv=1)
    bounds.update(kw)
    return ead.PagedBatch(OnGpu(page_table, device), OnGpu(torch.zeros(n + 1, dtype=torch.int32), device), OnGpu(lens, device), **bounds)


def test_overlapping_rows_of_a_page_table_are_refused():
    """An expanded row has a stride of 0: taken for rows `width` apart, sequence b's would be looked for b * width entries past its end."""
    row = torch.arange(4, dtype=torch.int32)[None]
    with pytest.raises(ValueError):
        batch_of(row.expand(3, -1))
    with pytest.raises(ValueError):
        batch_of(torch.arange(16, dtype=torch.int32).as_strided((3, 4), (2, 1)))
    assert batch_of(row.expand(3, -1).contiguous())._desc.table_stride == 4


def test_strides_of_page_tables():
    wide = torch.arange(40, dtype=torch.int32).view(4, 10)
    d = batch_of(wide[:, :6])._desc                          # columns of a wider table
    assert (d.table_width, d.table_stride) == (6, 10)
    d = batch_of(wide[::2, 2:])._desc                        # every second row
    assert (d.table_width, d.table_stride) == (8, 20)
    d = batch_of(wide[:1].expand(1, -1))._desc               # one sequence: its stride says nothing
    assert d.table_width == 10 and d.table_stride >= 10
    d = batch_of(torch.arange(3, dtype=torch.int32).as_strided((1, 3), (0, 1)))._desc
    assert d.table_width == 3 and d.table_stride >= 3


def cache_of(device="cuda:0", shape=(4, 2, 16, 64)):
    return ead.PagedCache(*(OnGpu(torch.zeros(shape, dtype=torch.bfloat16), device) for _ in range(2)))


def calls(cache, batch, k, q):
    return [lambda: cache.write(k, k, batch), lambda: cache.read(batch, out=(k, k)), lambda: cache.attention(q, batch, out=q)]


@pytest.mark.parametrize("where", [("cuda:1", "cuda:0", "cuda:0", 0), ("cuda:0", "cuda:1", "cuda:0", 0), ("cuda:0", "cuda:0", "cuda:1", 0),
                                   ("cuda:0", "cuda:0", "cuda:0", 1), ("cuda:1", "cuda:1", "cuda:1", 0)])
def test_tensors_of_different_devices_are_refused(monkeypatch, where):
    """Cache, batch, rows and the current device, whose stream the kernels are launched on, have to be one."""
    cache_on, batch_on, rows_on, current = where
    monkeypatch.setattr(paged, "_current_device", lambda: current, raising=False)
    monkeypatch.setattr(paged, "_stream_ptr", lambda: 0)
    table = torch.zeros(2, 3, dtype=torch.int32)
    k, q = OnGpu(torch.zeros(2, 2, 64, dtype=torch.bfloat16), rows_on), OnGpu(torch.zeros(2, 4, 64, dtype=torch.bfloat16), rows_on)
    for call in calls(cache_of(cache_on), batch_of(table, batch_on), k, q):
        with pytest.raises(ValueError):
            call()


def test_rows_on_the_host_are_refused(monkeypatch):
    monkeypatch.setattr(paged, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(paged, "_stream_ptr", lambda: 0)
    k, q = torch.zeros(2, 2, 64, dtype=torch.bfloat16), torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    for call in calls(cache_of(), batch_of(torch.zeros(2, 3, dtype=torch.int32)), k, q):
        with pytest.raises(ValueError):
            call()


def test_outputs_that_overlap_themselves_are_refused(monkeypatch):
    """An expanded output has several rows or heads in one place; inputs may be expanded."""
    monkeypatch.setattr(paged, "_current_device", lambda: 0)
    monkeypatch.setattr(paged, "_stream_ptr", lambda: 0)
    cache, batch = cache_of(), batch_of(torch.zeros(2, 3, dtype=torch.int32))
    q, k = (OnGpu(torch.zeros(2, n, 64, dtype=torch.bfloat16)) for n in (4, 2))
    flat = torch.zeros(1000, dtype=torch.bfloat16)
    for strides in ((0, 64, 1), (256, 0, 1), (256, 32, 1), (32, 128, 1)):
        with pytest.raises(ValueError):
            cache.attention(q, batch, out=OnGpu(flat.as_strided((2, 4, 64), strides)))
        with pytest.raises(ValueError):
            cache.read(batch, out=(k, OnGpu(flat.as_strided((2, 2, 64), strides))))
        with pytest.raises(ValueError):
            cache.read(batch, out=(OnGpu(flat.as_strided((2, 2, 64), strides)), k))
    # a dimension of 1 has no stride to speak of
    one = ead.PagedCache(*(OnGpu(torch.zeros(4, 1, 16, 64, dtype=torch.bfloat16)) for _ in range(2)))
    assert paged._outputs("out", OnGpu(flat.as_strided((2, 1, 64), (64, 0, 1))), one, 2, 1).row_stride == 64


def test_the_schedules_of_tests_are_their_threads_alone():
    """ead_test_paged changes how the calling thread's calls are cut; another thread's workspaces stay what its launches need."""
    L = ead.lib()
    L.ead_test_paged.argtypes = [C.c_double, C.c_int32]
    cache = paged.CacheDesc(1, 8, 16, 2, 64, 0x1000, 0x2000, None, None)
    batch = paged.BatchDesc(1, 1, 1, 1, 100, 8, 8, 0x3000, 0x4000, 0x5000)
    attn = paged.AttnDesc(4, 1, 0, 0, 0.125)

    def need():
        n = C.c_uint64(0)
        assert L.ead_paged_workspace(C.byref(cache), C.byref(batch), C.byref(attn), C.byref(n)) == 0
        return n.value

    plain, other = need(), []
    L.ead_test_paged(-1.0, 1)
    try:
        shares = need()
        t = threading.Thread(target=lambda: other.append(need()))
        t.start()
        t.join()
    finally:
        L.ead_test_paged(-1.0, 0)
    assert plain == 0 and shares > 0 and other == [plain] and need() == plain


def test_scales_whose_base_two_form_overflows_are_refused():
    """Scores are kept in bits: scale * log2(e) has to be a float32 too."""
    L = ead.lib()
    cache = paged.CacheDesc(1, 8, 16, 2, 64, 0x1000, 0x2000, None, None)
    batch = paged.BatchDesc(1, 1, 1, 1, 100, 8, 8, 0x3000, 0x4000, 0x5000)
    for scale, status in ((2.3e38, 0), (2.4e38, 1), (3.4e38, 1)):
        attn, n = paged.AttnDesc(4, 1, 0, 0, scale), C.c_uint64(0)
        assert L.ead_paged_workspace(C.byref(cache), C.byref(batch), C.byref(attn), C.byref(n)) == status


@pytest.mark.parametrize("bad", [2 ** 32 + 5, 2 ** 31, -2 ** 31 - 1])
def test_numbers_that_do_not_fit_are_refused(monkeypatch, bad):
    """The descriptors hold 32 bits, and ctypes would cut a larger number to them: 2^32 + 5 to 5."""
    monkeypatch.setattr(paged, "_current_device", lambda: 0)
    monkeypatch.setattr(paged, "_capturing", lambda: False)
    monkeypatch.setattr(paged, "_stream_ptr", lambda: 0)
    table = torch.zeros(2, 3, dtype=torch.int32)
    for name in ("max_kv", "rows", "max_q", "min_q"):
        with pytest.raises(ValueError):
            batch_of(table, **{name: bad})
    batch = batch_of(table)
    for name in ("window", "sinks"):
        with pytest.raises(ValueError):
            batch._plan(cache_of(), 4, *({"window": (bad, 0), "sinks": (0, bad)}[name]), 0.125, False, 0)
