"""Weights of positions that no row of a call sees (a window has passed them) are left as they are, bit for bit.  Tolerances are those of test_gpu_steps."""
import pytest
import torch

import paper_2502_06833_amd as ead
from test_gpu_paged import DEV, TYPES, Setup
from test_gpu_steps import check_weights, exact_weights

pytestmark = pytest.mark.gpu


def seen(s, window, sinks):
    """Which slots of the pool some row sees."""
    out = torch.zeros(s.cache.k_pages.shape[0], s.page, dtype=torch.bool, device=DEV)
    for b, (ql, kv) in enumerate(zip(s.q_lens, s.kv_lens)):
        j = torch.arange(kv, device=DEV)
        j = j[(j < sinks) | (kv - ql - j < window)] if ql else j[:0]
        out[torch.tensor(s.ids[b], dtype=torch.long, device=DEV)[j // s.page], j % s.page] = True
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (33, 0), (64, 5), (100, 32), (129, 300)])
@pytest.mark.parametrize("q_lens,kv_lens,heads,align", [([1, 0, 2], [700, 90, 2100], 8, 0), ([5, 1, 9], [700, 1, 333], 8, 0),
                                                       ([150, 1], [600, 900], 8, 0), ([150, 1], [600, 900], 8, 1),         # (the second with queries at odd places)
                                                       ([700, 40], [2900, 1333], 8, 0)])                                    # (several ranges of rows, joined)
def test_what_no_row_sees_keeps_its_weight(dtype, window, sinks, q_lens, kv_lens, heads, align):
    s = Setup(q_lens, kv_lens, 2, 64, dtype, 16, seed=window)
    s.write_all()
    q = s.queries(heads)
    if align:
        wide = torch.empty(q.shape[0], heads * 64 + 1, dtype=q.dtype, device=DEV)
        q = wide[:, 1:].unflatten(1, (heads, 64)).copy_(q)
    _, lse = s.cache.attention(q, s.batch, window=window, sinks=sinks, want_lse=True)
    mine = seen(s, window, sinks)[:, None].expand(-1, 2, -1)
    before = torch.rand(s.cache.k_pages.shape[:3], generator=s.g, device=DEV)
    # patterns that an addition of 0 would change: -0, NaN that signal
    patterns = torch.tensor([-2 ** 31, 0x7F800001, 0x7FA12345, -0x7FFFFF], dtype=torch.int32, device=DEV)
    odd = patterns[torch.randint(4, before.shape, generator=s.g, device=DEV)]
    before = torch.where(mine, before.view(torch.int32), odd).view(torch.float32)
    w = before.clone()
    s.cache.weigh(q, lse, s.batch, w, window=window, sinks=sinks)
    assert torch.equal(w.view(torch.int32)[~mine], before.view(torch.int32)[~mine])
    want, tol = exact_weights(s, q, lse, torch.where(mine, before, 0.0), window=window, sinks=sinks)
    assert bool(((w.double() - want).abs() <= tol)[mine].all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("q_lens", [[1, 1], [40, 3], [150, 120]])
def test_pages_that_went_to_another_sequence(dtype, q_lens):
    """A table that still names pages behind its window, which another sequence of the batch holds by now: the other one's weights are its own."""
    s = Setup(q_lens, [900, 700], 2, 64, dtype, 16, seed=6)
    s.write_all()
    q = s.queries(8)
    window, sinks = 130, 3
    _, lse = s.cache.attention(q, s.batch, window=window, sinks=sinks, want_lse=True)
    before = torch.rand(s.cache.k_pages.shape[:3], generator=s.g, device=DEV)
    want = before.clone()
    s.cache.weigh(q, lse, s.batch, want, window=window, sinks=sinks)
    check_weights(s, q, lse, want, before, window=window, sinks=sinks)
    behind = (900 - q_lens[0] - window) // 16                 # entries 1 .. behind - 1 of sequence 0 are seen by no row
    n = min(behind - 1, 44)
    stale = s.table.clone()
    stale[0, 1:1 + n] = s.table[1, :44].flip(0)[:n]           # sequence 1's last pages first, which its rows see
    batch = ead.PagedBatch(stale, s.batch.q_starts, s.batch.kv_lens, rows=sum(q_lens), max_q=q_lens[0], max_kv=900)
    for _ in range(5):
        w = before.clone()
        s.cache.weigh(q, lse, batch, w, window=window, sinks=sinks)
        assert torch.equal(w, want)
