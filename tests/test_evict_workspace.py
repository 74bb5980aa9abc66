"""The workspace of an eviction under budgets that no sequence reaches, without a GPU."""
import ctypes as C

import paper_2502_06833_amd as ead
from paper_2502_06833_amd import paged


def test_budgets_that_nothing_reaches_need_no_moves():
    L, n = ead.lib(), C.c_uint64(0)
    cache = paged.CacheDesc(1, 8, 16, 2, 64, 0x1000, 0x2000, None, None)
    batch = paged.BatchDesc(3, 4, 2, 1, 100, 8, 8, 0x3000, 0x4000, 0x5000)

    def need(keep, sinks=2, recent=8):
        ev = paged.EvictionDesc(keep, sinks, recent)
        assert L.ead_paged_evict_workspace(C.byref(cache), C.byref(batch), C.byref(ev), C.byref(n)) == 0
        return n.value

    counts = 32                                               # one of 4 bytes for each of 6 sequences and heads, to a multiple of 16
    assert need(99) == counts + 6 * 89 * 8                    # up to 100 positions: one may go
    assert need(100) == need(101) == need(2 ** 31 - 1) == counts
