"""Rotation, append, weighing, eviction and log probabilities at their edges: offsets past 32 bits, tables shorter than their sequences, the widest groups, other streams.
Tolerances are those of the tests that the helpers come from."""
import pytest
import torch

import paper_2502_06833_amd as ead
from test_gpu_logprobs import check, rows
from test_gpu_paged import DEV, F8, TYPES, Setup
from test_gpu_steps import check_rotated, check_weights, exact_weights, plain_kept, rotary_of, rows_of, weights_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, F8])
def test_pools_of_more_than_2_to_32_bytes(dtype):
    """The same sequence in a small pool and at the end of one whose vectors lie past 2^31 elements and 2^32 bytes."""
    n_kv, hd, page, n = 8, 64, 64, 300
    per = -(-n // page)
    n_pages = (2 ** 32 // (n_kv * page * hd * (2 if dtype == torch.bfloat16 else 1))) + 50
    big = ead.PagedCache.empty(n_pages, page, n_kv, hd, dtype)
    small = ead.PagedCache.empty(per, page, n_kv, hd, dtype)
    g = torch.Generator(device=DEV); g.manual_seed(0)
    rot = rotary_of(hd, g)
    got = []
    q, k, v = rows_of(n, (16, n_kv, n_kv), hd, torch.bfloat16, g)
    for cache, ids in ((big, [n_pages - 1 - 3 * i for i in range(per)]), (small, list(range(per)))):
        w = torch.empty(cache.k_pages.shape[:3], device=DEV)
        all_rows = ead.PagedBatch.of([ids], [n], [n])
        x = cache.append(q, k, v, all_rows, rot)
        _, lse = cache.attention(x, all_rows, want_lse=True)
        cache.weigh(x, lse, all_rows, w)                       # many rows
        first = w[ids].clone()
        one = ead.PagedBatch.of([ids], [1], [n])
        cache.weigh(x[-1:].contiguous(), lse[-1:].contiguous(), one, w)      # and one
        second = w[ids].clone()
        kept = cache.evict(ead.PagedBatch.of([ids], [0], [n]), w, 200, sinks=3, recent=20)
        held = ead.PagedBatch.of([ids], [200], [200])
        got.append([x, first, second, kept, *cache.read(held, torch.float32), w[ids].transpose(1, 2).reshape(-1, n_kv)[:200]])
    at = torch.arange(n, device=DEV)
    for name, a, b in zip(("q", "weights", "weights of one", "kept", "k", "v", "moved"), *got):
        if name.startswith("weights"):
            a, b = (t.transpose(1, 2).reshape(-1, n_kv)[at] for t in (a, b))
        assert torch.equal(a, b), name


def test_logits_of_more_than_2_to_31_elements():
    n, vocab = 15000, 151936
    x = torch.empty(n, vocab, dtype=torch.bfloat16, device=DEV)
    for i in range(0, n, 1000):
        x[i:i + 1000].normal_()
    t = torch.arange(n, device=DEV, dtype=torch.int32) * 10
    r = ead.logprobs(x, t, top=3)
    for i in (0, n // 2, n - 5):
        part = ead.logprobs(x[i:i + 5], t[i:i + 5], top=3)
        assert torch.equal(part.rank, r.rank[i:i + 5]) and torch.equal(part.top_tokens, r.top_tokens[i:i + 5])
        check(x[i:i + 5], type(r)(*(f[i:i + 5] for f in r)), t[i:i + 5], 3)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads", [(64, 1, 32), (64, 1, 128), (128, 2, 64)])
@pytest.mark.parametrize("q_lens", [[1, 1], [2, 1], [9, 30]])
def test_the_widest_groups(dtype, heads, q_lens):
    n_heads, n_kv, hd = heads
    s = Setup(q_lens, [77, 300], n_kv, hd, dtype, 16, seed=3)
    s.write_all()
    q = s.queries(n_heads)
    _, lse = s.cache.attention(q, s.batch, want_lse=True)
    w, before = weights_of(s)
    s.cache.weigh(q, lse, s.batch, w)
    check_weights(s, q, lse, w, before)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("q_lens", [[1], [60]])
def test_tables_shorter_than_their_sequences(dtype, q_lens):
    """What lies past the table is no one's; positions stay what the whole length makes them."""
    s = Setup(q_lens, [200], 2, 64, dtype, 16, seed=4)
    s.write_all()
    q = s.queries(6)
    _, lse = s.cache.attention(q, s.batch, want_lse=True)
    w, before = weights_of(s)
    short = ead.PagedBatch(s.table[:, :9].contiguous(), s.batch.q_starts, s.batch.kv_lens, rows=q_lens[0], max_q=q_lens[0], max_kv=200)     # 144 positions
    s.cache.weigh(q, lse, short, w)
    want, tol = exact_weights(s, q, lse, before, holes=[(0, p) for p in range(9, 13)])
    assert bool(((w.double() - want).abs() <= tol).all())
    # eviction sees a sequence of 144
    scores = torch.rand(w.shape, generator=s.g, device=DEV)
    k = s.cache.k_pages.view(torch.uint8).clone()
    kept = s.cache.evict(short, scores, 100, sinks=2, recent=30, weights=w)
    ids, at = torch.tensor(s.ids[0], device=DEV), torch.arange(144, device=DEV)
    for h in range(2):
        assert kept[0, h].tolist() == plain_kept(scores[ids[at // 16], h, at % 16].tolist(), 144, 100, 2, 30)
    for p in s.ids[0][9:]:
        assert torch.equal(s.cache.k_pages.view(torch.uint8)[p], k[p])


def test_sequences_longer_than_max_kv_are_left_as_they_are():
    s = Setup([0, 0], [150, 90], 2, 32, torch.float32, 16, seed=5)
    s.write_all()
    w = torch.rand(s.cache.k_pages.shape[:3], generator=s.g, device=DEV)
    low = ead.PagedBatch(s.table, s.batch.q_starts, s.batch.kv_lens, rows=0, max_q=0, max_kv=100)
    k, before = s.cache.k_pages.clone(), w.clone()
    kept = s.cache.evict(low, w, 60, recent=10)
    assert bool((kept[0] == -1).all()) and bool((kept[1] >= 0).all())
    for p in s.ids[0]:
        assert torch.equal(torch.nan_to_num(s.cache.k_pages[p]), torch.nan_to_num(k[p])) and torch.equal(w[p], before[p])


def test_other_streams():
    """Every call on a stream of its own, beside the others; the same as on one stream."""
    g = torch.Generator(device=DEV); g.manual_seed(6)
    rot = rotary_of(64, g)
    work = []
    for i in range(3):
        s = Setup([40, 1, 7], [140, 700, 7], 2, 64, (torch.bfloat16, F8, torch.float32)[i], 16, seed=i)
        s.write_all()
        work.append((s, rows_of(48, (8, 2, 2), 64, torch.float32 if i == 2 else torch.bfloat16, g), weights_of(s)[0], rows(5, 40001, torch.float32, seed=i)[0]))

    def one(s, qkv, w, logits, cache):
        x = cache.append(*qkv, s.batch, rot)
        out, lse = cache.attention(x, s.batch, want_lse=True)
        cache.weigh(x, lse, s.batch, w)
        kept = cache.evict(s.batch, w, 100, sinks=2, recent=30)
        return [x, out, lse, kept, w, *ead.logprobs(logits, top=9)[0:1], ead.logprobs(logits, top=9).top_tokens]

    def copy(c):
        return ead.PagedCache(*(t.clone() if t is not None else None for t in (c.k_pages, c.v_pages, c.k_scales, c.v_scales)))

    want = [one(s, qkv, w.clone(), logits, copy(s.cache)) for s, qkv, w, logits in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    for _ in range(5):
        got = []
        torch.cuda.synchronize()
        args = [(s, qkv, w.clone(), logits, copy(s.cache)) for s, qkv, w, logits in work]
        torch.cuda.synchronize()
        for stream, a in zip(streams, args):
            with torch.cuda.stream(stream):
                got.append(one(*a))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(torch.nan_to_num(x), torch.nan_to_num(y)) for x, y in zip(a, b))


def test_a_token_twice_and_rows_of_one_stride():
    """The same row and token several times over, as an expanded tensor."""
    x, _ = rows(1, 30000, torch.bfloat16, seed=8)
    t = torch.full((7,), 123, dtype=torch.int32, device=DEV)
    r = ead.logprobs(x.expand(7, -1), t, top=2)
    assert all(bool((f == f[:1]).all()) for f in r)
    check(x.expand(7, -1), r, t, 2)


def test_rotation_of_a_row_back_and_forth():
    """Turning by p and then by -p gives a vector back: the first turn's error of both of a pair, and the second's, of a pair that is twice as large at most."""
    g = torch.Generator(device=DEV); g.manual_seed(9)
    rot = ead.Rotary(128, 5e5)
    q, k = rows_of(50, (4, 2), 128, torch.float32, g)
    p = torch.randint(1 << 20, (50,), generator=g, device=DEV).to(torch.int32)
    a, b = rot(*rot(q, k, p), -p)
    for x, y in ((q, a), (k, b)):
        size = (x[..., :64].abs() + x[..., 64:].abs()).repeat(1, 1, 2)
        assert bool(((x - y).abs() <= 4 * 20 * 2.0 ** -24 * size).all())
    check_rotated(rot(q, k, p)[0], q, None, p, rot.inv_freq)


@pytest.mark.parametrize("n,keep,sinks,recent,ties", [(1 << 20, 600001, 5, 77, False), (1 << 20, 300000, 0, 250000, True), (200001, 100000, 16, 33, False), (70000, 35000, 1, 0, True),
                                                      (1 << 20, (1 << 20) - 3, 0, 1, True)])
def test_evict_the_longest_sequences(n, keep, sinks, recent, ties):
    """Sequences whose scores, and whose lists of moves, do not fit a workgroup's local memory."""
    page, per = 256, -(-n // 256)
    g = torch.Generator(device=DEV); g.manual_seed(n + keep)
    cache = ead.PagedCache.empty(per, page, 1, 32, F8)
    cache.k_pages.view(torch.uint8).random_(0, 256, generator=g), cache.v_pages.view(torch.uint8).random_(0, 256, generator=g)
    cache.k_scales.random_(1, 255, generator=g), cache.v_scales.random_(1, 255, generator=g)
    table = torch.randperm(per, generator=g, device=DEV).to(torch.int32)[None]
    batch = ead.PagedBatch.of(table, [0], [n])
    scores = torch.randn(per, 1, page, generator=g, device=DEV).exp()
    if ties:
        scores = (scores * 2).round()
    at = torch.arange(n, device=DEV)
    place = lambda p: (table[0].long()[p // page], 0, p % page)  # noqa: E731
    old = [t.view(torch.uint8)[place(at)].clone() for t in (cache.k_pages, cache.v_pages)] + [t[place(at)].clone() for t in (cache.k_scales, cache.v_scales, scores)]
    stay, cut = keep - sinks - recent, keep - recent
    chosen = torch.zeros(n, dtype=torch.bool, device=DEV)
    chosen[torch.sort(old[4][sinks:n - recent], descending=True, stable=True).indices[:stay] + sinks] = True
    want = at[:keep].clone()
    want[cut:] = at[n - recent:]
    free = (~chosen[:cut] & (at[:cut] >= sinks)).nonzero()[:, 0]
    late = chosen[cut:].nonzero()[:, 0] + cut
    assert free.numel() == late.numel() and (free.numel() > 40000 or keep > 10 ** 6 or n < 10 ** 6)
    want[free] = late
    kept = cache.evict(batch, scores, keep, sinks=sinks, recent=recent)
    assert torch.equal(kept[0, 0].long(), want)
    now = [t.view(torch.uint8)[place(at[:keep])] for t in (cache.k_pages, cache.v_pages)] + [t[place(at[:keep])] for t in (cache.k_scales, cache.v_scales, scores)]
    assert all(torch.equal(a, b[want]) for a, b in zip(now, old))
