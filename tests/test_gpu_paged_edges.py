"""The paged cache where calls leave the ordinary: tables that end before their sequences, workspaces and graphs, infinities and
magnitudes at the ends of their types.  Definitions, tolerances and set-ups are those of test_gpu_paged.py."""
import pytest
import torch

import paper_2502_06833_amd as ead
from test_gpu_paged import DEV, F8, TYPES, Setup, check_attention, exact_attention, way  # noqa: F401

pytestmark = pytest.mark.gpu


# (rows, positions, pages that the table has of 16 positions each)
SHORT = [(1, 33, 2), (1, 300, 2), (7, 36, 2), (5, 200, 12), (40, 70, 3), (150, 400, 20), (150, 180, 1)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("q_len,kv,width", SHORT)
def test_positions_past_the_table_are_holes(way, dtype, q_len, kv, width):
    """A table that ends before its sequence: the rest are holes.  Rows stay at their positions: nothing is written over others', nothing is
    read there, and what a row sees goes by its own position."""
    s = Setup([q_len, 2], [kv, 9], 2, 64, dtype, 16, seed=kv)
    s.write_all()
    short = ead.PagedBatch.of(s.table[:, :width], [q_len, 2], [kv, 9])
    past = [(0, p) for p in range(width, -(-kv // 16))]
    q = s.queries(6)
    for window, sinks in ((0, 0), (16 * width, 0), (16 * width + 1, 4), (20, 3), (3, 0), (2 ** 31 - 1, 2 ** 31 - 1)):
        got, lse = s.cache.attention(q, short, window=window, sinks=sinks, want_lse=True)
        check_attention(s, q, got, lse, exact_attention(s, q, window, sinks, holes=past))
    first = kv - q_len
    inside = torch.tensor([p < 16 * width for p in range(first, kv)] + [True, True], device=DEV)
    k, v = s.cache.read(short, torch.float32)
    whole = s.cache.read(s.batch, torch.float32)
    for part, all_ in zip((k, v), whole):
        assert bool((part[~inside] == 0).all()) and torch.equal(part[inside], all_[inside])
    # written: what is inside, and nothing else
    copies = [t.clone() if t is not None else None for t in (s.cache.k_pages, s.cache.v_pages, s.cache.k_scales, s.cache.v_scales)]
    full = ead.PagedCache(*copies)
    x = torch.randn(q_len + 2, 2, 64, generator=s.g, device=DEV)
    full.write(x, -x, s.batch)
    outside = s.table[0, width:].long()
    outside = outside[outside >= 0]
    for name in ("k_pages", "v_pages", "k_scales", "v_scales"):
        have, want = getattr(s.cache, name), getattr(full, name)
        if have is not None:
            want.view(torch.uint8)[outside] = have.view(torch.uint8)[outside]
    s.cache.write(x, -x, short)
    for name in ("k_pages", "v_pages", "k_scales", "v_scales"):
        if getattr(full, name) is not None:
            assert torch.equal(getattr(s.cache, name).view(torch.uint8), getattr(full, name).view(torch.uint8)), name


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("way_past", [2 ** 31 - 1, 2 ** 31 - 256, 10 ** 9])
def test_lengths_far_past_the_table(way, dtype, way_past):
    """Lengths up to the largest a device array holds: everything that the table has is seen, and nothing is written."""
    s = Setup([3], [48], 2, 32, dtype, 16, seed=1)
    s.write_all()
    lens = torch.tensor([way_past], dtype=torch.int32, device=DEV)
    far = ead.PagedBatch(s.table[:, :3], s.batch.q_starts, lens, rows=3, max_q=3, max_kv=way_past)
    q = s.queries(4)
    got, lse = s.cache.attention(q, far, want_lse=True)
    s.kv_lens = [51]                                          # three rows past the 48 positions see them all
    s.k, s.v = ([torch.cat([t[0], torch.zeros_like(t[0][:3])])] for t in (s.k, s.v))
    check_attention(s, q, got, lse, exact_attention(s, q, holes=[(0, 3)]))
    got, lse = s.cache.attention(q, far, window=40, sinks=5, want_lse=True)
    check_attention(s, q, got, lse, exact_attention(s, q, 1, 5, holes=[(0, 3)]))
    before = s.cache.k_pages.view(torch.uint8).clone()
    x = torch.ones(3, 2, 32, device=DEV)
    s.cache.write(x, x, far)
    assert torch.equal(s.cache.k_pages.view(torch.uint8), before)
    assert bool((s.cache.read(far)[0] == 0).all())


# ---- graphs
def _soiled_pool():
    """A graph pool whose free memory holds no zeros, and the graph that it belongs to."""
    pool, g = torch.cuda.graph_pool_handle(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, pool=pool):
        used = [torch.full((n,), 0x01010101, dtype=torch.int32, device=DEV) for n in [1 << 15] * 8 + [1 << 24] * 2]
    g.replay()
    torch.cuda.synchronize()
    del used
    return pool, g


def _captured(s, q, outs, pool=None):
    """A graph of one attention call for each of outs, on torch's own capture stream."""
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, pool=pool):
        for out in outs:
            s.cache.attention(q, s.batch, out=out)
    return g


@pytest.mark.parametrize("lens", [([1], [6000]), ([300], [5000])])
def test_first_calls_under_capture(way, lens):
    """No eager call before, two graphs of one batch on one capture stream, the second replayed first, then eager calls there and elsewhere:
    every one finds a workspace that was cleared for it."""
    def fresh():
        s = Setup(*lens, 1, 128, torch.bfloat16, 16, seed=5)
        s.write_all()
        return s, s.queries(8)

    s, q = fresh()
    want = s.cache.attention(q, s.batch)
    s, q = fresh()                                            # the same values, a batch that nothing was called for
    outs = [torch.full_like(q, 9.0) for _ in range(4)]
    (pool, zeroth), (pool2, zeroth2) = _soiled_pool(), _soiled_pool()
    first, second = _captured(s, q, outs[:2], pool), _captured(s, q, outs[2:], pool2)
    torch.cuda.synchronize()
    for _ in range(3):
        for graph, mine in ((second, outs[2:]), (first, outs[:2])):
            for o in outs:
                o.fill_(9.0)
            graph.replay()
            torch.cuda.synchronize()
            for o in mine:
                assert torch.equal(o, want)
            assert torch.equal(s.cache.attention(q, s.batch), want)
    s2, q2 = fresh()
    out = torch.full_like(q2, 9.0)
    pool, zeroth = _soiled_pool()
    graph = _captured(s2, q2, [out], pool)
    with torch.cuda.stream(torch.cuda.graph.default_capture_stream):           # eager on the capture stream, before any replay
        assert torch.equal(s2.cache.attention(q2, s2.batch), want)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_graphs_of_one_batch_replayed_side_by_side(way):
    """Graphs captured on one stream and replayed on others at the same time, beside eager calls on the capture stream."""
    s = Setup([1], [30000], 2, 128, torch.bfloat16, 16, seed=6)
    s.write_all()
    qs = [s.queries(16) for _ in range(3)]
    want = [s.cache.attention(q, s.batch) for q in qs]
    with torch.cuda.stream(torch.cuda.graph.default_capture_stream or torch.cuda.Stream()):
        s.cache.attention(qs[2], s.batch)
    outs = [[torch.zeros_like(q) for _ in range(4)] for q in qs[:2]]
    graphs = [_captured(s, q, o) for q, o in zip(qs, outs)]
    streams = [torch.cuda.Stream() for _ in graphs]
    torch.cuda.synchronize()
    for _ in range(50):
        eager = []
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        with torch.cuda.stream(torch.cuda.graph.default_capture_stream):
            for _ in range(4):
                eager.append(s.cache.attention(qs[2], s.batch))
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            for x in o:
                assert torch.equal(x, w)
                x.zero_()
        assert all(torch.equal(x, want[2]) for x in eager)
        torch.cuda.synchronize()


def test_a_graph_keeps_its_workspace(way):
    """The batch goes, the graph stays: its workspace lies in the graph's own memory."""
    s = Setup([1], [6000], 1, 128, torch.bfloat16, 16, seed=5)
    s.write_all()
    q = s.queries(8)
    want = s.cache.attention(q, s.batch)
    out = torch.zeros_like(q)
    graph = _captured(s, q, [out])
    lengths = s.batch.q_starts, s.batch.kv_lens               # these are the caller's to keep
    s.batch = None
    junk = [torch.full((1 << 22,), 0x01010101, dtype=torch.int32, device=DEV) for _ in range(20)]
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    assert all(bool((t == 0x01010101).all()) for t in junk) and len(lengths) == 2


# ---- infinities
def check_infinities(s, q, at, window=0, sinks=0):
    """V with an infinity in dimension 10 of position at[0] of every sequence, one of the other sign in 11, and both in 12 at at[0] and at[1]: a
    row that sees it has that infinity (NaN: both) there, whatever its weight, and everything else is as ever."""
    k, v = ([t.float().clone() for t in x] for x in (s.k, s.v))
    for x in v:
        for p in at:
            x[p, :, 10], x[p, :, 11] = torch.inf, -torch.inf
        x[at[0], :, 12], x[at[-1], :, 12] = torch.inf, -torch.inf if len(at) > 1 else torch.inf
    s.write_all(k=torch.cat(k), v=torch.cat(v))
    got, lse = s.cache.attention(q, s.batch, window=window, sinks=sinks, want_lse=True)
    s.v = [torch.where(torch.isfinite(x), x, 0.0) for x in s.v]
    out, z, mass = exact_attention(s, q, window, sinks)
    pos = torch.cat([torch.arange(kv - ql, kv, device=DEV) for ql, kv in zip(s.q_lens, s.kv_lens)])

    def sees(p):
        return (p <= pos) & ((pos - p < window) | (p < sinks) if window else pos >= 0)

    any_, first, last = torch.stack([sees(p) for p in at]).any(0), sees(at[0]), sees(at[-1])
    want = out.clone()
    want[any_, :, 10], want[any_, :, 11] = torch.inf, -torch.inf
    if len(at) == 1:
        want[first, :, 12] = torch.inf
    else:
        want[first & ~last, :, 12], want[last & ~first, :, 12], want[first & last, :, 12] = torch.inf, -torch.inf, torch.nan
    for d in (10, 11, 12):
        assert torch.equal(torch.nan_to_num(got[:, :, d].double(), 9e9, 8e8, 7e7) >= 7e7, torch.nan_to_num(want[:, :, d], 9e9, 8e8, 7e7) >= 7e7), d
        assert torch.equal(torch.isnan(got[:, :, d]), torch.isnan(want[:, :, d])) and torch.equal(torch.isinf(got[:, :, d]), torch.isinf(want[:, :, d]))
    fine = torch.isfinite(want)
    check_attention(s, q, torch.where(fine, got, 0.0), lse, (torch.where(fine, out, 0.0), z, mass))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("kv", [260, 390, 520, 650, 1300, 2100, 3400, 8190])
def test_an_infinity_outlives_the_join_of_parts(way, dtype, hd, kv):
    """The last position's, in a tile at the mask's edge: parts that are not there (their number is rounded up where they are read) add nothing."""
    s = Setup([1], [kv], 2, hd, dtype, 16, seed=kv)
    s.write_all()
    check_infinities(s, s.queries(4), [kv - 1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads", [(4, 2, 32), (6, 1, 128)])
@pytest.mark.parametrize("at", [[3], [97], [40, 90], [7, 97]])
@pytest.mark.parametrize("q_lens,kv_lens,window,sinks", [
    ([1, 1], [700, 131], 0, 0), ([1], [3000], 0, 0), ([5, 3], [700, 100], 0, 0), ([200], [700], 0, 0), ([200, 1], [200, 1500], 0, 0),
    ([1, 9], [150, 300], 100, 8), ([200, 60], [330, 300], 70, 60),
])
def test_infinities_that_rows_see(way, dtype, heads, at, q_lens, kv_lens, window, sinks):
    """In tiles that every row sees whole as at the edges."""
    n_heads, n_kv, hd = heads
    s = Setup(q_lens, kv_lens, n_kv, hd, dtype, 16, seed=at[0])
    s.write_all()
    check_infinities(s, s.queries(n_heads), at, window, sinks)


def test_infinities_in_long_contexts(way):
    s = Setup([200, 1], [4800, 5000], 1, 64, torch.bfloat16, 64, seed=2)
    s.write_all()
    check_infinities(s, s.queries(4), [3, 2000])


# ---- the ends of 8-bit exponents
@pytest.mark.parametrize("heads", [(4, 2, 32), (8, 2, 64), (6, 1, 128)])
@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1], [300, 40]), ([6], [129]), ([200], [250])])
@pytest.mark.parametrize("exponent", [1 + 127 - 80, 127, 127 + 90, 254])
def test_powers_of_two_to_the_largest(way, heads, q_lens, kv_lens, exponent):
    """V's codes are zeros and the smallest ones, its powers of two all the same: outputs are the same times that power, and zeros stay zeros."""
    n_heads, n_kv, hd = heads
    s = Setup(q_lens, kv_lens, n_kv, hd, F8, 16, seed=7)
    v = torch.randint(-1, 2, (sum(kv_lens), n_kv, hd), generator=s.g, device=DEV).float() * 2.0 ** -9
    v[:, :, 5] = 0.0
    s.write_all(v=v)
    s.cache.v_pages.copy_(torch.zeros_like(s.cache.v_pages))
    s.cache.v_scales.fill_(exponent)
    row = 0
    for ids, kv in zip(s.ids, kv_lens):
        for p in range(-(-kv // 16)):
            n = min(16, kv - 16 * p)
            s.cache.v_pages[ids[p], :, :n] = v[row:row + n].transpose(0, 1).to(F8)
            row += n
    s.v = [x.double() * 512 for x in v.split(kv_lens)]
    q = s.queries(n_heads, 1.5)
    got, lse = s.cache.attention(q, s.batch, want_lse=True)
    back = torch.tensor(2.0, dtype=torch.float64, device=DEV) ** (9 + 127 - exponent)
    assert bool((got[:, :, 5] == 0).all())
    ref = exact_attention(s, q)
    check_attention(s, q, (got.double() * back), lse, ref)


# ---- pages behind a window
def test_a_pair_in_a_pool_that_only_a_window_makes_do_with():
    """The pair of paged_pair.py with 15 pages for three sequences of up to 140 positions (9 pages each): with a window the run fits, token for
    token the one in a large pool, so no page went back that was still used; without one the pool runs out."""
    import paged_pair
    import synth_inputs as si
    weights = [si.model_weights_torch(s, 0, "cuda") for s in (si.TINY_S, si.TINY_L)]
    prompts = [si.prompt_np(0, f"pp{i}", n, si.TINY_S.vocab) for i, n in enumerate((5, 40, 23))]

    def run(n_pages, window, sinks, tau):
        models = [paged_pair.PagedModel(s, w, torch.float32, n_pages=n_pages, window=window, sinks=sinks) for s, w in zip((si.TINY_S, si.TINY_L), weights)]
        out, _, _ = paged_pair.run(models, prompts, [0, 2, 9], 100, tau=tau, d_min=4, piece=8)
        assert all(len(m.free) == n_pages for m in models)
        return out

    small = run(256, 20, 4, 1e30)
    tau = sorted(x for o in small for x in o["Hbar"])[150]
    wide, tight = run(256, 20, 4, tau), run(15, 20, 4, tau)
    for a, b in zip(wide, tight):
        assert a["tokens"] == b["tokens"] and a["model_id"] == b["model_id"] and a["H"] == b["H"]
    assert len({m for o in wide for m in o["model_id"]}) == 2
    with pytest.raises(RuntimeError, match="no free page"):
        run(15, 0, 0, tau)


# ---- terms of probabilities
def norm_error(got, out):
    return float((got.double() - out).norm() / out.norm())


# Rounding to bf16 is off by 2^-7 / sqrt(12) of the leading bit, 0.0016 of values spread over a binade, for the output's rounding alone; one bf16 term of
# each probability adds as much again, independent of it: 0.0023.  In between, and above:
TWO_TERMS, ONE_TERM = 0.0020, 0.0026


@pytest.mark.parametrize("dtype", [torch.bfloat16, F8])
@pytest.mark.parametrize("heads", [(8, 2, 64), (4, 1, 128), (4, 4, 32)])
def test_rounding_of_probabilities(dtype, heads):
    """Two terms for every row, whatever the other sequences' lengths or the bounds; one where the caller says so."""
    n_heads, n_kv, hd = heads
    lens = [700, 450, 300, 300, 260], [700, 2000, 4000, 9000, 5000]
    s = Setup(*lens, n_kv, hd, dtype, 64, seed=1)
    s.write_all()
    q = s.queries(n_heads, 1.5)
    generous = ead.PagedBatch(s.batch.page_table, s.batch.q_starts, s.batch.kv_lens, rows=sum(lens[0]), max_q=700, min_q=260, max_kv=10 ** 6)
    for window, sinks in ((0, 0), (4500, 100), (2000, 100)):
        out, z, _ = exact_attention(s, q, window, sinks)
        for batch in (s.batch, generous):
            for one_term in (False, True):
                got, lse = s.cache.attention(q, batch, window=window, sinks=sinks, want_lse=True, one_term=one_term)
                errors = [norm_error(a, b) for a, b in zip(got.split(lens[0]), out.split(lens[0]))]
                assert max(errors) <= (ONE_TERM if one_term else TWO_TERMS), errors
                assert float((lse.double() - z).abs().max()) <= 1e-5


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads", [(6, 2, 64), (8, 1, 128), (24, 1, 32)])
@pytest.mark.parametrize("q_lens,kv_lens,window,sinks", [
    ([130, 257], [130, 400], 0, 0), ([150, 1, 0], [600, 900, 5], 64, 33), ([200, 33], [333, 40], 129, 0), ([90], [2], 0, 0), ([700, 450], [5000, 4700], 0, 0),
])
def test_one_term(way, dtype, heads, q_lens, kv_lens, window, sinks):
    """A term is off by at most 2^-8 of itself (8 significant bits), and so is the output's rounding: 1.05 * 2^-8 (|out| + sum_j p_j |v_j|) + 1e-5."""
    n_heads, n_kv, hd = heads
    s = Setup(q_lens, kv_lens, n_kv, hd, dtype, 64, seed=1)
    s.write_all()
    q = s.queries(n_heads, 1.5)
    got, lse = s.cache.attention(q, s.batch, window=window, sinks=sinks, want_lse=True, one_term=True)
    out, z, mass = exact_attention(s, q, window, sinks)
    if dtype == torch.float32:                                # float32 pages take no terms
        return check_attention(s, q, got, lse, (out, z, mass))
    assert bool(((got.double() - out).abs() <= 1.05 * 2.0 ** -8 * (out.abs() + mass) + 1e-5).all())
    assert torch.equal(torch.isinf(lse), torch.isinf(z))
    f = torch.isfinite(z)
    assert float((lse.double() - z)[f].abs().max() if f.any() else 0.0) <= 1e-5


def test_one_term_of_infinities(way):
    """An infinity that a row sees is its output with one term too."""
    s = Setup([200], [700], 1, 128, torch.bfloat16, 16, seed=2)
    s.write_all()
    v = torch.cat(s.v).float()
    v[97, :, 10], v[97, :, 11] = torch.inf, -torch.inf
    s.write_all(k=torch.cat(s.k).float(), v=v)
    got = s.cache.attention(s.queries(4), s.batch, one_term=True)
    assert bool((got[:, :, 10] == torch.inf).all()) and bool((got[:, :, 11] == -torch.inf).all()) and bool(torch.isfinite(got[:, :, 12:]).all())
