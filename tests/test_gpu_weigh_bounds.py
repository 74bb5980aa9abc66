"""Weighing under bounds and lengths past 2^24 positions: page tables that are wide and mostly holes.  Tolerances are those of test_gpu_steps."""
import pytest
import torch

import paper_2502_06833_amd as ead
from test_gpu_paged import DEV, TYPES, Setup
from test_gpu_steps import check_weights, weights_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_kv", [1 << 28, (1 << 29) + 77, 0x7FFFFF00])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("q_lens", [[70, 33], [3, 1]])
def test_loose_bounds(max_kv, dtype, q_lens):
    """The bound says how large the grid may become, and nothing else."""
    page = 256
    s = Setup(q_lens, [300, 500], 1, 32, dtype, page, seed=1)
    s.write_all()
    q = s.queries(4)
    _, lse = s.cache.attention(q, s.batch, want_lse=True)
    w, before = weights_of(s)
    tight = before.clone()
    s.cache.weigh(q, lse, s.batch, tight)
    table = torch.full((2, -(-max_kv // page)), -1, dtype=torch.int32, device=DEV)
    table[:, :s.table.shape[1]] = s.table
    loose = ead.PagedBatch(table, s.batch.q_starts, s.batch.kv_lens, rows=sum(q_lens), max_q=q_lens[0], max_kv=max_kv)
    s.cache.weigh(q, lse, loose, w)
    assert torch.equal(w, tight)
    check_weights(s, q, lse, w, before)


def test_positions_past_the_grid():
    """A sequence of more than 2^24 positions, holes but for its first pages and those around and past the 2^24th: workgroups go on past their grid."""
    page, hd, n_kv, n_heads, rows = 256, 32, 2, 4, 70
    n = (1 << 24) + 700
    width = -(-n // page)
    at = [0, 1, (1 << 24) // page - 1, (1 << 24) // page, width - 1]              # the table's entries that are pages
    g = torch.Generator(device=DEV); g.manual_seed(2)
    cache = ead.PagedCache.empty(len(at) + 1, page, n_kv, hd, torch.float32)
    cache.k_pages.normal_(generator=g), cache.v_pages.normal_(generator=g)
    table = torch.full((1, width), -1, dtype=torch.int32)
    table[0, at] = torch.arange(1, len(at) + 1, dtype=torch.int32)
    batch = ead.PagedBatch.of(table.to(DEV), [rows], [n])
    q = torch.randn(rows, n_heads, hd, generator=g, device=DEV)
    lse = torch.rand(rows, n_heads, generator=g, device=DEV) + 2
    before = torch.rand(cache.k_pages.shape[:3], generator=g, device=DEV)
    w = before.clone()
    cache.weigh(q, lse, batch, w)
    assert torch.equal(w[0], before[0])
    i = torch.arange(n - rows, n, device=DEV)
    for p, entry in enumerate(at, 1):
        j = torch.arange(entry * page, entry * page + page, device=DEV)
        k = cache.k_pages[p].double().repeat_interleave(n_heads // n_kv, 0)      # [heads, slots, hd]
        a = torch.einsum("ihd,hjd->hij", q.double(), k) * hd ** -0.5
        mass = torch.einsum("ihd,hjd->hij", q.double().abs(), k.abs()) * hd ** -0.5
        z = lse.double().T[:, :, None]
        pay = torch.where((j[None] <= i[:, None])[None], torch.exp(a - z), 0.0)
        u = 2.0 ** -24
        off = pay * (u * ((hd + 2) * mass + 3 * a.abs() + 3 * z.abs()) + 4 * u + u * (rows * n_heads / n_kv / 4 + 8))
        pay, off = (t.view(n_kv, n_heads // n_kv, rows, page).sum((1, 2)) for t in (pay, off))
        want = torch.where(j[None] < n - rows, before[p].double(), 0.0) + pay
        want = torch.where(j[None] < n, want, before[p].double())                # slots past the sequence stay as they were
        assert bool(((w[p].double() - want).abs() <= off + u * want).all()), entry
