"""Rotation, append, weighing and eviction on the GPU against their definitions in 64 bits.

Tolerances, with u = 2^-24.  Rotation: a vector's factor 1 / sqrt(mean + eps) is a sum of 16 products to a lane and up to 3 exchanges, a root and a division, so off by less than
12 u; with the gain's two products an element by 14 u of itself; sines and cosines by 2 u, products and their sum by 2 u: 18 u (|a| + |b|), 20 taken.  bf16 outputs: half a
step more, 2^-8 of the value.  Weights: a score of n products is off by n u sum |q k| in the order of any hardware, the exponent by u of score and lse besides, each
exponential by 2 u, the sum by u for each addition."""
import math

import pytest
import torch

import paper_2502_06833_amd as ead
from test_gpu_paged import DEV, F8, HEADS, TYPES, Setup, exact_round

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


# ------------------------------------------------------------------------------------------ rotation
def exact_rotate(x, gain, positions, freq, interleaved=False, eps=1e-6):
    """(result, |a| + |b| of each element's pair) in 64 bits."""
    x = x.double()
    if gain is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * gain.double()
    r = 2 * freq.numel()
    angle = positions.double()[:, None, None] * freq.double()
    cos, sin = angle.cos(), angle.sin()
    out, size = x.clone(), x.abs()
    i, j = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    a, b = x[..., i], x[..., j]
    out[..., i], out[..., j] = a * cos - b * sin, b * cos + a * sin
    size[..., i] = size[..., j] = a.abs() + b.abs()
    return out, size


def check_rotated(got, x, gain, positions, freq, interleaved=False, eps=1e-6):
    want, size = exact_rotate(x, gain, positions, freq, interleaved, eps)
    tol = 20 * U * size + (2.0 ** -8 * (want.abs() + 20 * U * size) if got.dtype == torch.bfloat16 else 0.0) + 1e-37
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


def rows_of(n, heads, hd, dtype, g, fused=False, offset=0):
    if fused:
        flat = torch.randn(n, sum(heads) * hd + 13, generator=g, device=DEV).to(dtype)
        out, at = [], offset
        for h in heads:
            out.append(flat[:, at:at + h * hd].unflatten(1, (h, hd)))
            at += h * hd
        return out
    return [torch.randn(n, h, hd, generator=g, device=DEV).to(dtype) for h in heads]


def rotary_of(hd, g, norm=True, part=None, heads=None, **kw):
    gains = [1 + 0.3 * torch.randn(*((h,) if heads else ()), hd, generator=g, device=DEV) if norm else None for h in (heads or (0, 0))]
    return ead.Rotary(hd, 1e6, rotary_dim=part, q_gain=gains[0], k_gain=gains[1], **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hd,heads", [(32, (4, 4)), (64, (14, 2)), (128, (40, 8)), (128, (3, 1)), (64, (1, 0)), (32, (0, 5))])
@pytest.mark.parametrize("n", [1, 37, 700])
@pytest.mark.parametrize("norm,interleaved", [(True, False), (False, False), (True, True)])
def test_rotate(dtype, hd, heads, n, norm, interleaved):
    g = torch.Generator(device=DEV); g.manual_seed(hd + n)
    rot = rotary_of(hd, g, norm, interleaved=interleaved)
    q, k = rows_of(n, heads, hd, dtype, g)
    pos = torch.randint(100000, (n,), generator=g, device=DEV).to(torch.int32)
    for x, y, gain in zip((q, k), rot(q, k, pos), (rot.q_gain, rot.k_gain)):
        check_rotated(y, x, gain, pos, rot.inv_freq, interleaved)


@pytest.mark.parametrize("hd,part", [(32, 16), (64, 0), (64, 16), (128, 48), (128, 112)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_part_of_a_head_is_turned(hd, part, interleaved):
    g = torch.Generator(device=DEV); g.manual_seed(part)
    for norm in (True, False):
        rot = rotary_of(hd, g, norm, part, interleaved=interleaved)
        q, k = rows_of(29, (5, 2), hd, torch.float32, g)
        pos = torch.arange(29, dtype=torch.int32, device=DEV) * 1000
        out = rot(q, k, pos)
        for x, y, gain in zip((q, k), out, (rot.q_gain, rot.k_gain)):
            check_rotated(y, x, gain, pos, rot.inv_freq, interleaved)
            if not norm:
                assert torch.equal(y[..., part:], x[..., part:])


def test_far_and_negative_positions_and_given_frequencies():
    g = torch.Generator(device=DEV); g.manual_seed(1)
    freq = torch.rand(64, generator=g, device=DEV, dtype=torch.float64) * 3
    rot = ead.Rotary(128, inv_freq=freq)
    pos = torch.tensor([0, 1, -1, 2 ** 20 + 1, 2 ** 24 + 1, -2 ** 24 - 3, 10 ** 8], dtype=torch.int32, device=DEV)
    q, k = rows_of(7, (3, 2), 128, torch.float32, g)
    for x, y in zip((q, k), rot(q, k, pos)):
        # an angle of 3e8 radians is off by 2^-53 of itself in the reference too: 4e-8
        check_rotated(y, x, None, pos, rot.inv_freq)


def test_gains_per_head_strides_and_in_place():
    g = torch.Generator(device=DEV); g.manual_seed(2)
    for offset in (0, 1, 8):
        for dtype in (torch.float32, torch.bfloat16):
            rot = rotary_of(64, g, heads=(6, 2), eps=1e-5)
            q, k = rows_of(21, (6, 2), 64, dtype, g, fused=True, offset=offset)
            pos = torch.arange(21, dtype=torch.int32, device=DEV)
            qc, kc = q.clone(), k.clone()
            out = rot(q, k, pos)
            for x, y, gain in zip((q, k), out, (rot.q_gain, rot.k_gain)):
                check_rotated(y, x, gain, pos, rot.inv_freq, eps=1e-5)
            big = torch.full((21, 9, 70), 7.0, device=DEV, dtype=dtype)
            view = (big[:, 1:7, 3:67], torch.empty_like(k))
            rot(q, k, pos, out=view)
            assert torch.equal(view[0], out[0]) and torch.equal(view[1], out[1])
            assert bool((big[:, 0] == 7).all()) and bool((big[:, 7:] == 7).all()) and bool((big[:, :, :3] == 7).all()) and bool((big[:, :, 67:] == 7).all())
            rot(q, k, pos, out=(q, k))
            assert torch.equal(q, out[0]) and torch.equal(k, out[1]) and not torch.equal(q, qc) and not torch.equal(k, kc)


def test_vectors_of_zeros_and_not_finite_ones():
    g = torch.Generator(device=DEV); g.manual_seed(3)
    rot = rotary_of(32, g)
    q, k = rows_of(4, (2, 2), 32, torch.float32, g)
    q[0] = 0.0
    q[1, 0, 3] = math.nan
    y, _ = rot(q, k, torch.arange(4, dtype=torch.int32, device=DEV))
    assert bool((y[0] == 0).all()) and bool(torch.isnan(y[1, 0]).all()) and bool(torch.isfinite(y[1, 1]).all()) and bool(torch.isfinite(y[2:]).all())


# ------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hd,heads,page", [(32, (3, 3), 16), (64, (14, 2), 32), (128, (8, 8), 256), (128, (5, 1), 64)])
@pytest.mark.parametrize("part,norm", [(1, True), (1, False), (2, True)])
def test_append(dtype, src, hd, heads, page, part, norm):
    """Queries by the definition; the pages hold bit for bit what `write` puts there of the same keys turned in float32, and nothing else changes."""
    s = Setup([1, 0, 17, 5, 40], [1, 9, 17, 77, 301], heads[1], hd, dtype, page, seed=3)
    rot = rotary_of(hd, s.g, norm, hd // part)
    n = sum(s.q_lens)
    q, k, v = rows_of(n, (*heads, heads[1]), hd, src, s.g, fused=True, offset=8)
    pos = torch.cat([torch.arange(kv - ql, kv) for ql, kv in zip(s.q_lens, s.kv_lens)]).to(torch.int32).to(DEV)
    out = s.cache.append(q, k, v, s.batch, rot)
    check_rotated(out, q, rot.q_gain, pos, rot.inv_freq)
    got = [t.clone().view(torch.uint8) for t in (s.cache.k_pages, s.cache.v_pages)] + [t.clone() for t in (s.cache.k_scales, s.cache.v_scales) if t is not None]
    s.fill(float("nan"))
    turned = rot(q.float(), k.float(), pos)[1]
    s.cache.write(turned, v.float(), s.batch)
    want = [t.view(torch.uint8) for t in (s.cache.k_pages, s.cache.v_pages)] + [t for t in (s.cache.k_scales, s.cache.v_scales) if t is not None]
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # positions of the caller's: other angles, the same places
    far = pos * 3 + 1000
    out = s.cache.append(q, k, v, s.batch, rot, positions=far)
    check_rotated(out, q, rot.q_gain, far, rot.inv_freq)
    rk, rv = s.cache.read(s.batch, torch.float32)
    assert torch.equal(rk.double(), exact_round(rot(q.float(), k.float(), far)[1], dtype)[0]) and torch.equal(rv.double(), exact_round(v.float(), dtype)[0])


def test_append_leaves_alone_what_is_not_its_own():
    """Rows of no sequence, holes, positions below 0 and past the table."""
    cache = ead.PagedCache.empty(6, 16, 2, 64, torch.bfloat16)
    cache.k_pages.fill_(7.0), cache.v_pages.fill_(7.0)
    g = torch.Generator(device=DEV); g.manual_seed(4)
    rot = rotary_of(64, g)
    table = torch.tensor([[0, 99], [-1, 2], [3, 4]], dtype=torch.int32, device=DEV)
    starts = torch.tensor([0, 20, 24, 30], dtype=torch.int32, device=DEV)
    batch = ead.PagedBatch(table, starts, torch.tensor([20, 18, 2], dtype=torch.int32, device=DEV), rows=33, max_q=20, max_kv=32)
    q, k, v = rows_of(33, (4, 2, 2), 64, torch.bfloat16, g)
    out = torch.full_like(q, 5.0)
    cache.append(q, k, v, batch, rot, out=out)
    assert bool((out[30:] == 5).all()) and not bool((out[:30] == 5).all(-1).any())
    mine = torch.zeros(6, 16, dtype=torch.bool, device=DEV)
    mine[0] = True                          # sequence 0: 20 positions, the second page is none
    mine[2, :2] = True                      # sequence 1: positions 14 .. 17, the first page is a hole
    mine[3, :2] = True                      # sequence 2: six rows, two positions
    touched = (cache.k_pages != 7).any(-1).any(1)
    assert torch.equal(touched, mine) and torch.equal((cache.v_pages != 7).any(-1).any(1), mine)
    k2 = rot(q.float(), k.float(), torch.cat([torch.arange(20), torch.arange(14, 18), torch.arange(-4, 2), torch.zeros(3)]).to(torch.int32).to(DEV))[1].bfloat16()
    assert torch.equal(cache.k_pages[3][:, :2].transpose(0, 1), k2[28:30]) and torch.equal(cache.v_pages[3][:, :2].transpose(0, 1), v[28:30])


# ------------------------------------------------------------------------------------------ weighing
def exact_weights(s, q, lse, before, window=0, sinks=0, scale=None, holes=()):
    """Pages of weights in 64 bits, and how far off each may be."""
    out, tol = before.double().clone(), torch.zeros(before.shape, dtype=torch.float64, device=DEV)
    row, group = 0, q.shape[1] // s.n_kv
    scale = s.hd ** -0.5 if scale is None else scale
    for b, (ql, kv) in enumerate(zip(s.q_lens, s.kv_lens)):
        x, z = q[row:row + ql].double(), lse[row:row + ql].double(); row += ql
        if ql == 0:
            continue
        i = torch.arange(kv - ql, kv, device=DEV)[:, None]; j = torch.arange(kv, device=DEV)[None]
        see = j <= i
        if window:
            see = see & ((i - j < window) | (j < sinks))
        k = torch.nan_to_num(s.k[b]).repeat_interleave(group, 1)
        a = torch.einsum("ihd,jhd->hij", x, k) * scale
        mass = torch.einsum("ihd,jhd->hij", x.abs(), k.abs()) * scale
        zz = z.T[:, :, None]
        p = torch.where(see[None] & (zz != -math.inf), torch.exp(a - torch.where(zz == -math.inf, 0.0, zz)), 0.0)
        off = p * (U * ((s.hd + 2) * mass + 3 * a.abs() + 3 * torch.where(torch.isfinite(zz), zz.abs(), 0.0)) + 4 * U + U * (ql * group / 4 + 8))
        p, off = (t.view(s.n_kv, group, ql, kv).sum((1, 2)) for t in (p, off))
        at = torch.arange(kv, device=DEV)
        ids = torch.tensor(s.ids[b], device=DEV)
        for hb, hole in holes:
            if hb == b:
                at = at[at // s.page != hole]
        page, slot = ids[at // s.page], at % s.page
        old = torch.where(at < kv - ql, before.double()[page, :, slot].T, 0.0)
        out[page, :, slot] = (old + p[:, at]).T
        tol[page, :, slot] = (off[:, at] + U * (old + p[:, at])).T
    return out, tol


def check_weights(s, q, lse, weights, before, **kw):
    want, tol = exact_weights(s, q, lse, before, **kw)
    err = (weights.double() - want).abs()
    assert bool((err <= tol).all()), float((err - tol).max())


def weights_of(s):
    w = torch.rand(s.cache.k_pages.shape[:3], generator=s.g, device=DEV)
    return w, w.clone()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("q_lens,kv_lens,page", [
    ([1, 1, 1, 1], [1, 16, 33, 1000], 16),                  # decode
    ([1], [5000], 64),                                      # decode, one long sequence
    ([3, 0, 5, 1, 8], [3, 40, 200, 0 + 1, 129], 32),        # a few rows, some sequences without
    ([17, 40, 1], [17, 300, 77], 16),                       # pieces of prompts
    ([130, 257], [130, 400], 256),
    ([33, 1, 513], [900, 1500, 513], 128),
])
def test_weigh(dtype, heads, q_lens, kv_lens, page):
    n_heads, n_kv, hd = heads
    s = Setup(q_lens, kv_lens, n_kv, hd, dtype, page, seed=11)
    s.write_all()
    q = s.queries(n_heads, 1.5)
    _, lse = s.cache.attention(q, s.batch, want_lse=True)
    w, before = weights_of(s)
    assert s.cache.weigh(q, lse, s.batch, w) is w
    check_weights(s, q, lse, w, before)
    # all that is paid is what there was to pay: 1 for every row and head
    for b, (ql, kv) in enumerate(zip(q_lens, kv_lens)):
        at = torch.arange(kv, device=DEV)
        page, slot = torch.tensor(s.ids[b], dtype=torch.long, device=DEV)[at // s.page], at % s.page
        old = torch.where(at < kv - ql, before.double()[page, :, slot].T, 0.0)
        assert ql == 0 or abs(float((w.double()[page, :, slot].T - old).sum()) / (ql * n_heads) - 1) < 1e-3
    again = before.clone()
    s.cache.weigh(q, lse, s.batch, again)
    assert torch.equal(again, w)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (31, 4), (64, 33), (100, 0), (5000, 7), (33, 5000)])
@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1, 1], [700, 40, 2100]), ([5, 1, 9], [700, 1, 333]), ([150, 1], [600, 900])])
def test_weigh_window_and_sinks(dtype, window, sinks, q_lens, kv_lens):
    s = Setup(q_lens, kv_lens, 2, 64, dtype, 16, seed=window)
    s.write_all()
    q = s.queries(8)
    _, lse = s.cache.attention(q, s.batch, window=window, sinks=sinks, want_lse=True)
    w, before = weights_of(s)
    s.cache.weigh(q, lse, s.batch, w, window=window, sinks=sinks)
    check_weights(s, q, lse, w, before, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("q_lens", [[1, 1], [40, 90]])
def test_weigh_holes_nan_and_rows_that_pay_nothing(dtype, q_lens):
    """Holes keep what their pages' memory held; stale slots (NaN) and keys of other positions that are NaN change nothing; a row whose lse is -inf pays nothing."""
    s = Setup(q_lens, [100, 333], 2, 64, dtype, 16, seed=9)
    s.write_all()
    q = s.queries(6)
    _, lse = s.cache.attention(q, s.batch, want_lse=True)
    lse[0, 1] = -math.inf
    s.table[1, 3] = -1
    # a key that is NaN: its own weight alone
    page, slot = s.ids[1][5], 7
    if dtype != F8:
        s.cache.k_pages[page, 0, slot] = math.nan
    w, before = weights_of(s)
    s.cache.weigh(q, lse, s.batch, w)
    want, tol = exact_weights(s, q, lse, before, holes=[(1, 3)])
    bad = torch.zeros(w.shape, dtype=torch.bool, device=DEV)
    if dtype != F8:
        bad[page, 0, slot] = True
    assert bool(torch.isnan(w[bad]).all())
    assert bool(((w.double() - want).abs() <= tol)[~bad].all())
    assert torch.equal(w[s.ids[1][3]], before[s.ids[1][3]])


@pytest.mark.parametrize("offset", [0, 1, 8])
def test_weigh_strided_queries_and_scale(offset):
    for dtype in TYPES:
        s = Setup([7, 33], [20, 33], 2, 64, dtype, 32, seed=5)
        s.write_all()
        t = torch.float32 if dtype == torch.float32 else torch.bfloat16
        flat = torch.randn(40, 6 * 64 + 13, generator=s.g, device=DEV).to(t)
        q = flat[:, offset:offset + 6 * 64].unflatten(1, (6, 64))
        _, lse = s.cache.attention(q, s.batch, want_lse=True, scale=0.31)
        w, before = weights_of(s)
        s.cache.weigh(q, lse, s.batch, w, scale=0.31)
        check_weights(s, q, lse, w, before, scale=0.31)


# ------------------------------------------------------------------------------------------ eviction
def plain_kept(score, n, keep, sinks, recent):
    """Which position lies where, from one sequence's and head's scores (a list)."""
    if n <= keep:
        return list(range(n)) + [-1] * (keep - n)
    value = lambda j: -math.inf if math.isnan(score[j]) else score[j]  # noqa: E731
    order = sorted(range(sinks, n - recent), key=lambda j: (math.isnan(score[j]), -value(j), j))
    chosen = set(order[:keep - sinks - recent])
    cut = keep - recent
    late = iter(sorted(j for j in chosen if j >= cut))
    return [i if i < sinks or i in chosen else next(late) for i in range(cut)] + list(range(n - recent, n))


def check_evict(s, scores, keep, sinks, recent, weights=None, lens=None):
    lens = s.kv_lens if lens is None else lens
    old = [t.clone() for t in (s.cache.k_pages.view(torch.uint8).view(*s.cache.k_pages.shape[:3], -1), s.cache.v_pages.view(torch.uint8).view(*s.cache.k_pages.shape[:3], -1))]
    old += [t.clone() for t in (s.cache.k_scales, s.cache.v_scales) if t is not None]
    moved = scores if weights is None else weights
    old.append(moved.clone())
    want = [t.clone() for t in old]
    before = scores.clone()
    kept = s.cache.evict(s.batch, scores, keep, sinks=sinks, recent=recent, weights=weights)
    assert kept.shape == (len(lens), s.n_kv, keep)
    for b, n in enumerate(lens):
        ids = torch.tensor(s.ids[b], dtype=torch.long, device=DEV)
        at = torch.arange(n, device=DEV)
        for h in range(s.n_kv):
            sc = before[ids[at // s.page], h, at % s.page].tolist()
            k = plain_kept(sc, n, keep, sinks, recent)
            assert kept[b, h].tolist() == k, (b, h)
            src = torch.tensor([i for i in k if i >= 0], dtype=torch.long, device=DEV)
            dst = torch.arange(src.numel(), device=DEV)
            for t, o in zip(want, old):
                t[ids[dst // s.page], h, dst % s.page] = o[ids[src // s.page], h, src % s.page]
    now = [s.cache.k_pages.view(torch.uint8).view(*s.cache.k_pages.shape[:3], -1), s.cache.v_pages.view(torch.uint8).view(*s.cache.k_pages.shape[:3], -1)]
    now += [t for t in (s.cache.k_scales, s.cache.v_scales) if t is not None] + [moved]
    # slots past the cut may hold anything of the sequence's, and hold what they held
    for t, x in zip(now, want):
        assert torch.equal(torch.nan_to_num(t.float()), torch.nan_to_num(x.float()))
    if weights is not None:
        assert torch.equal(torch.nan_to_num(scores), torch.nan_to_num(before))
    return kept


def scores_of(s, ties=False):
    w = torch.randn(s.cache.k_pages.shape[:3], generator=s.g, device=DEV).exp()
    return (w * 2).round() / 2 if ties else w


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hd,page", [(32, 16), (64, 32), (128, 256)])
@pytest.mark.parametrize("lens,keep,sinks,recent", [
    ([1, 2, 3, 4], 1, 0, 0), ([1, 2, 3, 4], 1, 0, 1), ([5, 4, 3], 2, 1, 1), ([40, 33, 17, 16], 16, 4, 5), ([100, 99, 64, 63, 65], 64, 0, 0),
    ([300, 500, 129, 7], 128, 16, 100), ([300, 500, 129, 7], 128, 0, 128), ([300, 500, 129, 7], 128, 128, 0), ([777, 2049], 700, 3, 600), ([1000], 999, 1, 7),
])
@pytest.mark.parametrize("ties", [False, True])
def test_evict(dtype, hd, page, lens, keep, sinks, recent, ties):
    s = Setup([0] * len(lens), lens, 3, hd, dtype, page, seed=keep)
    s.write_all()
    w = scores_of(s, ties)
    check_evict(s, w, keep, sinks, recent)


@pytest.mark.parametrize("n,keep,sinks,recent", [(5000, 1200, 4, 100), (13000, 12500, 0, 3000), (20001, 9000, 16, 33), (40000, 30000, 1, 0)])
def test_evict_long_sequences(n, keep, sinks, recent):
    s = Setup([0, 0], [n, n - 700], 2, 64, torch.bfloat16, 64, seed=n)
    s.write_all()
    w = scores_of(s, True)
    other = torch.rand(w.shape, generator=s.g, device=DEV)
    check_evict(s, w, keep, sinks, recent, weights=other)


def test_evict_scores_of_all_kinds():
    """Zeros of both signs, negative numbers, infinities, NaN, subnormal ones, all the same."""
    lens = [200, 200, 200, 150]
    s = Setup([0] * 4, lens, 2, 32, torch.float32, 16, seed=1)
    s.write_all()
    w = scores_of(s)
    special = torch.tensor([0.0, -0.0, 1e-45, -1e-45, math.inf, -math.inf, math.nan, -1.0, 1.0, 3.4e38, -3.4e38], device=DEV)
    for p in s.ids[0]:
        w[p] = special[torch.randint(special.numel(), w[p].shape, generator=s.g, device=DEV)]
    for p in s.ids[1]:
        w[p] = math.nan
    for p in s.ids[2]:
        w[p] = -0.0
        w[p, :, ::2] = 0.0
    check_evict(s, w, 64, 2, 9)


def test_evict_holes():
    s = Setup([0], [96], 1, 32, torch.float32, 16, seed=2)
    s.write_all()
    w = scores_of(s) + 1
    k = s.cache.k_pages.clone()
    s.table[0, 1] = -1                                        # positions 16 .. 31: no place, a score of 0
    kept = s.cache.evict(s.batch, w, 48, sinks=0, recent=16)
    of = kept[0, 0].tolist()
    assert not any(16 <= j < 32 for j in of[:16]) and of[32:] == list(range(80, 96))
    for i, j in enumerate(of):
        if i // 16 == 1:
            continue                                          # nothing is written there
        assert torch.equal(s.cache.k_pages[s.ids[0][i // 16], 0, i % 16], k[s.ids[0][j // 16], 0, j % 16])
    assert torch.equal(s.cache.k_pages[s.ids[0][1]], k[s.ids[0][1]])


# ------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype", TYPES)
def test_a_run_within_a_budget(dtype):
    """Prompt, then steps of append, attention, weigh and now and then evict over two sequences, captured step by step in none; the same in 64 bits beside it."""
    n_heads, n_kv, hd, page, keep, sinks, recent = 6, 2, 64, 16, 40, 2, 8
    g = torch.Generator(device=DEV); g.manual_seed(0)
    cache = ead.PagedCache.empty(16, page, n_kv, hd, dtype)
    rot = rotary_of(hd, g)
    t = torch.float32 if dtype == torch.float32 else torch.bfloat16
    weights = cache.new_weights()
    weights.fill_(math.nan)                                   # new positions start from nothing, whatever is there
    table = torch.arange(16, dtype=torch.int32, device=DEV).view(2, 8)
    held, text = [0, 0], [0, 0]
    ref_k, ref_v, ref_w = ([[torch.zeros(0, hd, dtype=torch.float64, device=DEV) for _ in range(n_kv)] for _ in range(2)] for _ in range(3))
    ref_w = [[torch.zeros(0, dtype=torch.float64, device=DEV) for _ in range(n_kv)] for _ in range(2)]
    for step, lens in enumerate([(37, 30)] + [(1, 1)] * 25 + [(5, 1)] + [(1, 1)] * 10):
        n = sum(lens)
        held = [h + m for h, m in zip(held, lens)]
        batch = ead.PagedBatch.of(table, lens, held)
        pos = torch.cat([torch.arange(x, x + m) for x, m in zip(text, lens)]).to(torch.int32).to(DEV)
        text = [x + m for x, m in zip(text, lens)]
        q, k, v = rows_of(n, (n_heads, n_kv, n_kv), hd, t, g)
        q2 = cache.append(q, k, v, batch, rot, positions=pos)
        out, lse = cache.attention(q2, batch, want_lse=True)
        cache.weigh(q2, lse, batch, weights)
        kk, vv = exact_round(rot(q.float(), k.float(), pos)[1], dtype)[0], exact_round(v.float(), dtype)[0]
        row = 0
        for b, m in enumerate(lens):
            for c in range(n_kv):
                ref_k[b][c] = torch.cat([ref_k[b][c], kk[row:row + m, c]])
                ref_v[b][c] = torch.cat([ref_v[b][c], vv[row:row + m, c]])
                ref_w[b][c] = torch.cat([ref_w[b][c], torch.zeros(m, dtype=torch.float64, device=DEV)])
                see = torch.arange(held[b], device=DEV)[None] <= torch.arange(held[b] - m, held[b], device=DEV)[:, None]
                for h in range(c * 3, c * 3 + 3):
                    a = torch.where(see, q2[row:row + m, h].double() @ ref_k[b][c].T * hd ** -0.5, -math.inf)
                    p = torch.softmax(a, 1)
                    ref_w[b][c] += p.sum(0)
                    o = p @ ref_v[b][c]
                    tol = 2e-6 if t == torch.float32 else 2.0 ** -7
                    assert float((out[row:row + m, h].double() - o).abs().max()) <= tol * max(1.0, float(ref_v[b][c].abs().max()))
            row += m
        for b in range(2):
            at = torch.arange(held[b], device=DEV)
            for c in range(n_kv):
                got = weights[table[b].long()[at // page], c, at % page].double()
                assert float((got - ref_w[b][c]).abs().max()) <= 1e-4 * (1 + step)
        if max(held) > keep + 5:
            kept = cache.evict(batch, weights, keep, sinks=sinks, recent=recent)
            for b in range(2):
                for c in range(n_kv):
                    of = kept[b, c][kept[b, c] >= 0].long()
                    assert of.numel() == min(held[b], keep)
                    ref_k[b][c], ref_v[b][c], ref_w[b][c] = ref_k[b][c][of], ref_v[b][c][of], ref_w[b][c][of]
                    if held[b] > keep:
                        assert of[:sinks].tolist() == list(range(sinks)) and of[-recent:].tolist() == list(range(held[b] - recent, held[b]))
            held = [min(x, keep) for x in held]
    assert max(text) > keep + 30


def test_a_captured_step():
    """append, attention, weigh and evict in one graph, replayed on new rows with eager work between; every replay against the eager calls."""
    n_heads, n_kv, hd, page = 8, 2, 64, 16
    g = torch.Generator(device=DEV); g.manual_seed(5)
    rot = rotary_of(hd, g)
    table = torch.arange(20, dtype=torch.int32, device=DEV).view(2, 10)
    lens = [150, 141]
    batch = ead.PagedBatch.of(table, [3, 1], lens)
    start = ead.PagedCache.empty(20, page, n_kv, hd, torch.bfloat16)
    start.k_pages.normal_(generator=g), start.v_pages.normal_(generator=g)
    w0 = torch.rand(20, n_kv, page, generator=g, device=DEV)
    q, k, v = rows_of(4, (n_heads, n_kv, n_kv), hd, torch.bfloat16, g)

    def fresh():
        return ead.PagedCache(start.k_pages.clone(), start.v_pages.clone()), w0.clone()

    def step(cache, w):
        x = cache.append(q, k, v, batch, rot)
        out, lse = cache.attention(x, batch, want_lse=True)
        cache.weigh(x, lse, batch, w)
        return x, out, lse, cache.evict(batch, w, 96, sinks=4, recent=20)

    cache, w = fresh()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(cache, w)
    for i in range(4):
        for x in (q, k, v):
            x.normal_(generator=g)
        cache.k_pages.copy_(start.k_pages), cache.v_pages.copy_(start.v_pages), w.copy_(w0)
        graph.replay()
        other, w2 = fresh()
        want = step(other, w2)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert torch.equal(cache.k_pages, other.k_pages) and torch.equal(cache.v_pages, other.v_pages) and torch.equal(w, w2)
