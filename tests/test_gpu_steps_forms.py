"""The forms that large calls of the steps around attention take, each reached by its rule in csrc/paged_rules.hpp: four heads to a group of lanes in rotation and append (bf16 heads of 64
and 128; the others stay with one, for many rows too), several tiles to a wave in weighing, wide and narrow workgroups that move in eviction.  Tolerances are those of test_gpu_steps."""
import pytest
import torch

import paper_2502_06833_amd as ead
from test_gpu_paged import DEV, F8, TYPES, Setup, exact_round
from test_gpu_steps import check_evict, check_rotated, check_weights, exact_weights, rotary_of, rows_of, weights_of

pytestmark = pytest.mark.gpu
WIDE = 4 * 256 * 1024                                         # lanes past which heads go four to a group


def wide_rows(heads, hd, more):
    return WIDE // (heads * (hd // 16)) + more


# ------------------------------------------------------------------------------------------ four heads to a group
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hd,heads", [(32, (7, 2)), (64, (14, 2)), (128, (9, 5)), (128, (4, 0)), (64, (0, 3))])
@pytest.mark.parametrize("kind", ["norm", "plain", "interleaved", "per head", "part", "odd places"])
def test_rotate_many_rows(dtype, hd, heads, kind):
    g = torch.Generator(device=DEV); g.manual_seed(hd + sum(heads))
    n = wide_rows(sum(heads), hd, 3)
    rot = rotary_of(hd, g, kind != "plain", hd // 2 if kind == "part" else None, heads if kind == "per head" and all(heads) else None, interleaved=kind in ("interleaved", "part"))
    q, k = rows_of(n, heads, hd, dtype, g, fused=kind in ("odd places", "per head"), offset=1 if kind == "odd places" else 8)
    pos = torch.randint(-10, 100000, (n,), generator=g, device=DEV).to(torch.int32)
    out = rot(q, k, pos)
    for x, y, gain in zip((q, k), out, (rot.q_gain, rot.k_gain)):
        if x.numel():
            check_rotated(y, x, gain, pos, rot.inv_freq, kind in ("interleaved", "part"))
    # the rows of a small call, bit for bit: which form takes a row changes nothing
    some = torch.randint(n, (50,), generator=g, device=DEV)
    few = rot(q[some].contiguous(), k[some].contiguous(), pos[some].contiguous())
    assert torch.equal(few[0], out[0][some]) and torch.equal(few[1], out[1][some])
    # into places of the caller's, then in place
    big = torch.full((n, heads[0] + 2, hd + 8), 7.0, device=DEV, dtype=dtype)
    rot(q, k, pos, out=(big[:, 1:1 + heads[0], 3:3 + hd], torch.empty_like(k)))
    assert torch.equal(big[:, 1:1 + heads[0], 3:3 + hd], out[0]) and bool((big[:, 0] == 7).all()) and bool((big[:, -1] == 7).all())
    assert bool((big[..., :3] == 7).all()) and bool((big[..., 3 + hd:] == 7).all())
    rot(q, k, pos, out=(q, k))
    assert torch.equal(q, out[0]) and torch.equal(k, out[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hd,heads,page", [(32, (7, 3), 16), (64, (14, 2), 32), (128, (9, 5), 256)])
@pytest.mark.parametrize("kind", ["norm", "plain", "interleaved", "per head", "odd places"])
def test_append_many_rows(dtype, src, hd, heads, page, kind):
    """Prompts and pieces of them beside single rows, a sequence without any, and rows of none at the end."""
    n = wide_rows(heads[0] + 2 * heads[1], hd, 100)
    q_lens = [1, 0, n // 2, 1, n - n // 2 - 20]
    s = Setup(q_lens, [300, 9, q_lens[2], 77, q_lens[4] + 1000], heads[1], hd, dtype, page, seed=3)
    rot = rotary_of(hd, s.g, kind != "plain", None, heads if kind == "per head" else None, interleaved=kind == "interleaved")
    rows, used = n, sum(q_lens)
    q, k, v = rows_of(rows, (*heads, heads[1]), hd, src, s.g, fused=True, offset=1 if kind == "odd places" else 8)
    pos = torch.cat([torch.arange(kv - ql, kv) for ql, kv in zip(s.q_lens, s.kv_lens)] + [torch.zeros(rows - used, dtype=torch.long)]).to(torch.int32).to(DEV)
    batch = ead.PagedBatch(s.table, s.batch.q_starts, s.batch.kv_lens, rows=rows, max_q=max(q_lens), max_kv=max(s.kv_lens))
    out = torch.full(q.shape, 5.0, device=DEV, dtype=src)
    s.cache.append(q, k, v, batch, rot, out=out)
    check_rotated(out[:used], q[:used], rot.q_gain, pos[:used], rot.inv_freq, kind == "interleaved")
    assert bool((out[used:] == 5).all())
    pools = lambda: [t.view(torch.uint8) for t in (s.cache.k_pages, s.cache.v_pages)] + [t for t in (s.cache.k_scales, s.cache.v_scales) if t is not None]  # noqa: E731
    got = [t.clone() for t in pools()]
    s.fill(float("nan"))
    s.cache.write(rot(q.float(), k.float(), pos)[1], v.float(), batch)
    assert all(torch.equal(a, b) for a, b in zip(got, pools()))
    far = pos * 3 + 1000
    s.cache.append(q, k, v, batch, rot, positions=far, out=q if kind == "norm" else out)
    if kind == "norm":
        out = q
    want = rot(q.float(), k.float(), far)[1][:used]
    rk, rv = s.cache.read(s.batch, torch.float32)
    assert torch.equal(rk.double(), exact_round(want, dtype)[0]) and torch.equal(rv.double(), exact_round(v[:used].float(), dtype)[0])


# ------------------------------------------------------------------------------------------ several tiles to a wave
def loosely(s, max_kv=1 << 20):
    """The same batch under a bound that gives every wave eight tiles."""
    table = torch.full((s.table.shape[0], -(-max_kv // s.page)), -1, dtype=torch.int32, device=DEV)
    table[:, :s.table.shape[1]] = s.table
    assert s.table.shape[0] * s.n_kv * (max_kv // 128) > 8 * 8 * 256
    return ead.PagedBatch(table, s.batch.q_starts, s.batch.kv_lens, rows=s.batch.rows, max_q=max(s.q_lens), max_kv=max_kv)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("rows,group", [(1, 5), (3, 10), (4, 16)])               # one block of 16 rows, two, four (of float32 with heads of 128: the simple kernel)
@pytest.mark.parametrize("page", [16, 32, 256])
@pytest.mark.parametrize("window,sinks", [(0, 0), (700, 40)])
def test_weigh_with_several_tiles_to_a_wave(dtype, hd, rows, group, page, window, sinks):
    """Waves whose rings of tiles go round several times, end early, and end in the middle of a tile."""
    s = Setup([rows, 1, 0, rows], [1, 1025 + 31, 50, 2900], 2, hd, dtype, page, seed=hd + rows) if rows == 1 else \
        Setup([rows, 1, 0, rows], [rows + 129, 1024, 50, 2900], 2, hd, dtype, page, seed=hd + rows)
    s.write_all()
    q = s.queries(2 * group, 1.5)
    _, lse = s.cache.attention(q, s.batch, window=window, sinks=sinks, want_lse=True)
    w, before = weights_of(s)
    s.cache.weigh(q, lse, loosely(s), w, window=window, sinks=sinks)
    check_weights(s, q, lse, w, before, window=window, sinks=sinks)
    tight = before.clone()
    s.cache.weigh(q, lse, s.batch, tight, window=window, sinks=sinks)           # a tile to a wave: the same sums
    assert torch.equal(w, tight)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hd", [32, 128])
def test_weigh_holes_and_a_row_that_pays_nothing_with_several_tiles(dtype, hd):
    s = Setup([1, 2], [2000, 2777], 2, hd, dtype, 16, seed=9)
    s.write_all()
    q = s.queries(6)
    _, lse = s.cache.attention(q, s.batch, want_lse=True)
    lse[1, 4] = -float("inf")
    holes = [(1, 0), (1, 1), (1, 40), (1, 63), (0, 124)]
    for b, p in holes:
        s.table[b, p] = -1 if p & 1 else 10 ** 6
    w, before = weights_of(s)
    s.cache.weigh(q, lse, loosely(s), w)
    want, tol = exact_weights(s, q, lse, before, holes=holes)
    assert bool(((w.double() - want).abs() <= tol).all())
    for b, p in holes:
        assert torch.equal(w[s.ids[b][p]], before[s.ids[b][p]])


@pytest.mark.parametrize("dtype", TYPES)
def test_many_sequences_of_many_lengths(dtype):
    """As many sequences as give every wave several tiles by the rule itself, decode rows and catch-ups."""
    lens = [1 + (i * 2477) % 4100 for i in range(80)]
    s = Setup([1 + (i % 3 if n > 3 else 0) for i, n in enumerate(lens)], lens, 4, 64, dtype, 32, seed=1)
    s.write_all()
    q = s.queries(16)
    _, lse = s.cache.attention(q, s.batch, want_lse=True)
    w, before = weights_of(s)
    s.cache.weigh(q, lse, s.batch, w)
    check_weights(s, q, lse, w, before)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 4)])
def test_a_piece_of_a_prompt_beside_decode_rows(dtype, window, sinks):
    """One piece of 1500 rows beside 63 single rows, in append and weigh: every sequence as if it were alone."""
    n_heads, n_kv, hd = 8, 2, 64
    q_lens, kv_lens = [1] * 30 + [1500] + [1] * 33, [17 + 29 * i for i in range(30)] + [2600] + [900 + i for i in range(33)]
    s = Setup(q_lens, kv_lens, n_kv, hd, dtype, 16, seed=4)
    s.write_all()
    g = s.g
    t = torch.float32 if dtype == torch.float32 else torch.bfloat16
    rot = rotary_of(hd, g)
    x, k, v = rows_of(sum(q_lens), (n_heads, n_kv, n_kv), hd, t, g)
    q = s.cache.append(x, k, v, s.batch, rot)
    pos = torch.cat([torch.arange(n - m, n) for m, n in zip(q_lens, kv_lens)]).to(torch.int32).to(DEV)
    kk, row = exact_round(rot(x.float(), k.float(), pos)[1], dtype)[0], 0
    for b, m in enumerate(q_lens):
        s.k[b] = torch.cat([s.k[b][:kv_lens[b] - m], kk[row:row + m]]); row += m
    check_rotated(q, x, rot.q_gain, pos, rot.inv_freq)
    _, lse = s.cache.attention(q, s.batch, window=window, sinks=sinks, want_lse=True)
    w, before = weights_of(s)
    s.cache.weigh(q, lse, s.batch, w, window=window, sinks=sinks)
    check_weights(s, q, lse, w, before, window=window, sinks=sinks)


# ------------------------------------------------------------------------------------------ eviction
@pytest.mark.parametrize("dtype", [torch.bfloat16, F8])
@pytest.mark.parametrize("n_seqs", [70, 150])                                    # pieces of vectors, and whole ones, moved down by 256 threads
def test_evict_many_sequences(dtype, n_seqs):
    lens = [90 + (i * 37) % 90 for i in range(n_seqs)]
    s = Setup([0] * n_seqs, lens, 2, 128, dtype, 16, seed=n_seqs)
    s.write_all()
    w = torch.randn(s.cache.k_pages.shape[:3], generator=s.g, device=DEV).exp()
    check_evict(s, w, 96, 3, 70)


def test_evict_many_long_sequences():
    """Many free places in many sequences: places shared by few workgroups each, and the last positions by 256 threads."""
    lens = [1700 + 13 * i for i in range(66)]
    s = Setup([0] * 66, lens, 2, 64, torch.bfloat16, 64, seed=2)
    s.write_all()
    w = torch.randn(s.cache.k_pages.shape[:3], generator=s.g, device=DEV).exp()
    check_evict(s, w, 1000, 0, 300)


@pytest.mark.parametrize("keep", [301, 100000])
def test_evict_budgets_that_nothing_reaches(keep):
    lens = [300, 1, 0, 77]
    s = Setup([0] * 4, lens, 2, 32, torch.float32, 16, seed=2)
    s.write_all()
    w = torch.rand(s.cache.k_pages.shape[:3], generator=s.g, device=DEV)
    pools = [s.cache.k_pages.view(torch.uint8), s.cache.v_pages.view(torch.uint8), w]
    before = [t.clone() for t in pools]
    kept = s.cache.evict(s.batch, w, keep, sinks=2, recent=9)
    at = torch.arange(keep, device=DEV)
    for b, n in enumerate(lens):
        assert torch.equal(kept[b].long(), torch.where(at < n, at, -1).expand(2, -1))
    assert all(torch.equal(a, b) for a, b in zip(pools, before))
