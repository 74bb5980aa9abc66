"""The paged cache on the GPU: write, read and attention against their definitions in float64.

Tolerances.  Write and read round once (or not at all): codes, exponents and values are compared exactly.  Attention's
float32 path sums at most a few thousand products of magnitude about 1 in float32: 2e-6 of the largest output is several
times their rounding.  The bf16 path rounds its output to bf16 (relative 2^-9 at most); probabilities enter as one bf16
term at the least (2^-9 of each summand at most, of either sign), so an element is off by at most 2^-9 |out| + 2^-9
sum_j p_j |v_j|: the bound used is 1.05 times that plus 1e-5.  Log-sum-exps are float32 throughout: 1e-5 absolute for values up to
some tens (exponents rounded at 2^-24 of a score of a few tens)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2502_06833_amd as ead

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F8 = torch.float8_e4m3fn


def two_to(e):
    """2^e, exact (a power function is not, in the last bit)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def exact_round(x, dtype):
    """What a cache of that type holds for x (float32 or bf16 vectors), as float64, and the exponents."""
    if dtype == F8:
        x = x.double()
        amax = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1, keepdim=True)
        m, e = torch.frexp(amax / 448)
        e = torch.where(m > 0.5, e, e - 1).clamp(-126, 127)           # the smallest e with amax <= 448 * 2^e
        e = torch.where(amax == 0, torch.full_like(e, -126), e)
        y = x * two_to(-e)
        step = two_to(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
        r = torch.round(y / step) * step                      # half to even
        r = torch.where(torch.isfinite(x), r, torch.nan)
        return r * two_to(e), (e[..., 0] + 127).to(torch.uint8)
    return x.to(dtype).double(), None


@pytest.fixture(params=["as ever", "many rows", "shares"])
def way(request):
    """The kernels and schedules that a call's size would not choose by itself: k_paged_chunk for all sequences of more than 32 or 64
    rows per KV head however little work they are, and equal shares of the keys however short the contexts."""
    L = ead.lib()
    L.ead_test_paged.argtypes = [C.c_double, C.c_int32]
    L.ead_test_paged(0.0 if request.param == "many rows" else -1.0, 1 if request.param == "shares" else 0)
    yield request.param
    L.ead_test_paged(-1.0, 0)


class Setup:
    """Sequences of the given lengths in a shuffled pool; `pos[b]` of the pool's pages hold position-major values k, v."""

    def __init__(self, q_lens, kv_lens, n_kv, hd, dtype, page=16, seed=0, extra_pages=3, stale=float("nan"), wide=1):
        self.q_lens, self.kv_lens, self.n_kv, self.hd, self.dtype, self.page = q_lens, kv_lens, n_kv, hd, dtype, page
        g = torch.Generator(device=DEV); g.manual_seed(seed)
        self.g = g
        per = [-(-n // page) for n in kv_lens]
        n_pages = sum(per) + extra_pages
        perm = torch.randperm(n_pages, generator=g, device=DEV).tolist()
        self.ids, at = [], 0
        for n in per:
            self.ids.append(perm[at:at + n]); at += n
        self.cache = ead.PagedCache.empty(n_pages, page, n_kv, hd, dtype, DEV)
        self.fill(stale)
        self.table = torch.full((len(per), max(per + [1]) + wide), -1, dtype=torch.int32)
        for b, ids in enumerate(self.ids):
            self.table[b, :len(ids)] = torch.tensor(ids, dtype=torch.int32)
        self.table = self.table.to(DEV)
        self.batch = ead.PagedBatch.of(self.table, q_lens, kv_lens)
        self.k, self.v = [], []

    def fill(self, stale):
        for t in (self.cache.k_pages, self.cache.v_pages):
            if self.dtype == F8:
                t.view(torch.uint8).fill_(0x7F if stale != stale else 0)
            else:
                t.fill_(stale)
        for t in (self.cache.k_scales, self.cache.v_scales):
            if t is not None:
                t.fill_(255 if stale != stale else 127)

    def write_all(self, src=torch.float32, k=None, v=None):
        """Every position of every sequence written by one call; self.k / self.v hold the values kept, float64 [kv, n_kv, hd]."""
        n = sum(self.kv_lens)
        k = torch.randn(n, self.n_kv, self.hd, generator=self.g, device=DEV).to(src) if k is None else k
        v = torch.randn(n, self.n_kv, self.hd, generator=self.g, device=DEV).to(src) if v is None else v
        self.cache.write(k, v, ead.PagedBatch.of(self.table, self.kv_lens, self.kv_lens))
        self.k = list(exact_round(k, self.dtype)[0].split(self.kv_lens))
        self.v = list(exact_round(v, self.dtype)[0].split(self.kv_lens))

    def queries(self, n_heads, scale=1.0):
        t = torch.float32 if self.dtype == torch.float32 else torch.bfloat16
        return (scale * torch.randn(sum(self.q_lens), n_heads, self.hd, generator=self.g, device=DEV)).to(t)


def exact_attention(s, q, window=0, sinks=0, scale=None, holes=()):
    """(out, lse, sum_j p_j |v_j|) in float64."""
    out, lse, mass = [], [], []
    row, group = 0, q.shape[1] // s.n_kv
    scale = s.hd ** -0.5 if scale is None else scale
    for b, (ql, kv) in enumerate(zip(s.q_lens, s.kv_lens)):
        x = q[row:row + ql].double(); row += ql
        i = torch.arange(kv - ql, kv, device=DEV)[:, None]; j = torch.arange(kv, device=DEV)[None]
        see = j <= i
        if window:
            see = see & ((i - j < window) | (j < sinks))
        for hb, page in holes:
            if hb == b:
                see = see & (j // s.page != page)
        k, v = s.k[b].repeat_interleave(group, 1), s.v[b].repeat_interleave(group, 1)
        a = torch.einsum("ihd,jhd->hij", x, torch.nan_to_num(k) if kv else k) * scale
        a = torch.where(see[None], a, -math.inf)
        top = a.amax(-1, keepdim=True) if kv else torch.full((q.shape[1], ql, 1), -math.inf, device=DEV, dtype=torch.float64)
        p = torch.exp(a - torch.where(top == -math.inf, 0.0, top))
        z = p.sum(-1, keepdim=True)
        p = p / torch.where(z > 0, z, 1.0)
        out.append(torch.einsum("hij,jhd->ihd", p, v)); mass.append(torch.einsum("hij,jhd->ihd", p, v.abs()))
        lse.append((top + torch.log(z))[..., 0].T)
    return torch.cat(out), torch.cat(lse), torch.cat(mass)


def check_attention(s, q, got, lse, ref):
    out, z, mass = ref
    err = (got.double() - out).abs()
    if q.dtype == torch.float32:
        assert err.max() <= 2e-6 * max(1.0, float(out.abs().max())), float(err.max())
    else:
        bound = 1.05 * 2.0 ** -9 * (out.abs() + mass) + 1e-5
        assert bool((err <= bound).all()), float((err - bound).max())
    if lse is not None:
        assert torch.equal(torch.isinf(lse), torch.isinf(z)), "rows that see nothing"
        f = torch.isfinite(z)
        assert float((lse.double() - z)[f].abs().max() if f.any() else 0.0) <= 1e-5


TYPES = [torch.float32, torch.bfloat16, F8]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hd,n_kv,page", [(32, 3, 16), (64, 2, 32), (128, 8, 256), (128, 1, 64)])
def test_write_then_read(dtype, src, hd, n_kv, page):
    s = Setup([1, 0, 17, 5, 40], [1, 9, 17, 77, 301], n_kv, hd, dtype, page, seed=3)
    n = sum(s.q_lens)
    k = (torch.randn(n, n_kv, hd, generator=s.g, device=DEV) * torch.exp(6 * torch.randn(n, n_kv, 1, generator=s.g, device=DEV))).to(src)
    v = torch.randn(n, n_kv, hd, generator=s.g, device=DEV).to(src)
    k[0, 0] = 0.0
    before = s.cache.k_pages.clone().view(torch.uint8)
    s.cache.write(k, v, s.batch)
    for t in (torch.float32, torch.bfloat16):
        rk, rv = s.cache.read(s.batch, t)
        for r, x in ((rk, k), (rv, v)):
            want = exact_round(x, dtype)[0]
            if dtype == torch.float32 and t == torch.bfloat16:
                want = want.float().to(t).double()
            assert torch.equal(r.double(), want)
    # nothing else was written
    mine = torch.zeros(s.cache.k_pages.shape[0], page, dtype=torch.bool)
    for b, (ql, kv) in enumerate(zip(s.q_lens, s.kv_lens)):
        for p in range(kv - ql, kv):
            mine[s.ids[b][p // page], p % page] = True
    same = (s.cache.k_pages.view(torch.uint8) == before).view(s.cache.k_pages.shape[0], n_kv, page, -1).all(-1).all(1).cpu()
    assert bool(same[~mine].all())
    if dtype == F8:
        e = exact_round(k, dtype)[1]
        row = 0
        for b, (ql, kv) in enumerate(zip(s.q_lens, s.kv_lens)):
            for p in range(kv - ql, kv):
                assert torch.equal(s.cache.k_scales[s.ids[b][p // page], :, p % page], e[row]); row += 1


@pytest.mark.parametrize("scale", [2.0 ** -126, 2.0 ** -100, 1.0, 2.0 ** 100, 2.0 ** 119])
def test_eight_bit_codes_over_the_range(scale):
    """Every e4m3 code survives a round trip at scales from the smallest to the largest, and halves go to even."""
    codes = torch.arange(256, dtype=torch.uint8, device=DEV)
    vals = codes.view(F8).float()
    vals = vals[torch.isfinite(vals)]
    halves = (vals[1:126] + vals[:125]) / 2
    x = torch.cat([vals, halves, -halves])
    x = torch.nn.functional.pad(x, (0, -x.numel() % 31)).view(-1, 31)
    x = torch.cat([torch.full_like(x[:, :1], 448.0), x], 1) * scale            # 448 in every vector: the scale is known
    n = x.shape[0]
    s = Setup([n], [n], 1, 32, F8)
    s.cache.write(x.view(n, 1, 32), x.view(n, 1, 32), s.batch)
    k, v = s.cache.read(s.batch, torch.float32)
    want = (x / scale).to(F8).float() * scale
    keep = want.abs() >= 2.0 ** -126                                           # below, float32 values of the read are subnormal
    assert torch.equal(k.view(n, 32)[keep], want[keep]) and torch.equal(v.view(n, 32)[keep], want[keep])
    assert float((k.view(n, 32) - want).abs().max()) <= 2.0 ** -126


@pytest.mark.parametrize("dtype", TYPES)
def test_not_finite_values_stay_visible(dtype):
    s = Setup([4], [4], 2, 64, dtype)
    x = torch.randn(4, 2, 64, generator=s.g, device=DEV)
    x[1, 0, 5], x[2, 1, 63], x[3, 0, 0] = math.inf, math.nan, -math.inf
    s.cache.write(x, x, s.batch)
    k, _ = s.cache.read(s.batch, torch.float32)
    assert torch.equal(torch.isfinite(k), torch.isfinite(x))
    want = exact_round(x, dtype)[0]
    fine = torch.isfinite(x)
    assert torch.equal(k.double()[fine], want[fine])


@pytest.mark.parametrize("dtype,src", [(torch.bfloat16, torch.bfloat16), (F8, torch.bfloat16), (torch.float32, torch.float32)])
@pytest.mark.parametrize("offset", [0, 1, 8])
def test_strided_rows(way, dtype, src, offset):
    """Q, K and V as slices of one projection's output, at offsets that do and do not keep 16-byte alignment."""
    n_heads, n_kv, hd = 6, 2, 64
    s = Setup([7, 33], [20, 33], n_kv, hd, dtype, 32, seed=5)
    s.write_all()
    n = sum(s.q_lens)
    flat = torch.randn(n, (n_heads + 2 * n_kv) * hd + 13, generator=s.g, device=DEV).to(src)
    part = lambda first, heads: flat[:, offset + first * hd:offset + (first + heads) * hd].unflatten(1, (heads, hd))  # noqa: E731
    q, k, v = part(0, n_heads), part(n_heads, n_kv), part(n_heads + n_kv, n_kv)
    s.cache.write(k, v, s.batch)
    rk, rv = s.cache.read(s.batch, src)
    assert torch.equal(rk.double(), exact_round(k, dtype)[0]) and torch.equal(rv.double(), exact_round(v, dtype)[0])
    big = torch.full((n, 2 * n_heads, hd + 3), 7.0, device=DEV, dtype=src)
    view = big[:, 1::2, 1:hd + 1]
    got = s.cache.attention(q, s.batch, out=view)
    assert torch.equal(got, s.cache.attention(q.contiguous(), s.batch))
    assert bool((big[:, ::2] == 7).all()) and bool((big[:, :, 0] == 7).all()) and bool((big[:, :, hd + 1:] == 7).all())
    kv = torch.full((n, n_kv + 1, hd + 1), 7.0, device=DEV, dtype=src), torch.full((n, n_kv, hd), 7.0, device=DEV, dtype=src)
    s.cache.read(s.batch, out=(kv[0][:, 1:, 1:], kv[1]))
    assert torch.equal(kv[0][:, 1:, 1:], rk) and torch.equal(kv[1], rv) and bool((kv[0][:, 0] == 7).all())


# (query heads, KV heads, head_dim)
HEADS = [(4, 4, 32), (14, 2, 64), (8, 1, 128), (40, 8, 128), (24, 1, 32)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("q_lens,kv_lens,page", [
    ([1, 1, 1, 1], [1, 16, 33, 1000], 16),                  # decode
    ([1], [5000], 64),                                      # decode, one long sequence
    ([3, 0, 5, 1, 8], [3, 40, 200, 0 + 1, 129], 32),        # a few rows, some sequences without
    ([17, 40, 1], [17, 300, 77], 16),                       # pieces of prompts
    ([130, 257], [130, 400], 256),
])
def test_attention(way, dtype, heads, q_lens, kv_lens, page):
    n_heads, n_kv, hd = heads
    s = Setup(q_lens, kv_lens, n_kv, hd, dtype, page, seed=11)
    s.write_all()
    q = s.queries(n_heads, 1.5)
    got, lse = s.cache.attention(q, s.batch, want_lse=True)
    check_attention(s, q, got, lse, exact_attention(s, q))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (31, 4), (64, 33), (100, 0), (5000, 7), (33, 5000)])
@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1, 1], [700, 40, 2100]), ([5, 1, 9], [700, 1, 333]), ([150, 1], [600, 900])])
def test_window_and_sinks(way, dtype, window, sinks, q_lens, kv_lens):
    s = Setup(q_lens, kv_lens, 2, 64, dtype, 16, seed=window)
    s.write_all()
    q = s.queries(6, 1.5)
    got, lse = s.cache.attention(q, s.batch, window=window, sinks=sinks, want_lse=True)
    check_attention(s, q, got, lse, exact_attention(s, q, window, sinks))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [3, 40, 200])
def test_rows_before_the_first_position_see_nothing(way, dtype, n):
    """More rows than positions: the first rows are at positions below 0; and sequences that hold nothing at all."""
    s = Setup([n, n, 2], [2, 0, 0], 2, 64, dtype, 16)
    s.write_all()
    q = s.queries(4)
    got, lse = s.cache.attention(q, s.batch, want_lse=True)
    empty = torch.ones(2 * n + 2, dtype=torch.bool, device=DEV)
    empty[n - 2:n] = False
    assert bool((got[empty] == 0).all()) and bool((lse[empty] == -math.inf).all())
    check_attention(s, q, got, lse, exact_attention(s, q))
    k, v = s.cache.read(s.batch, torch.float32)
    assert bool((k[empty] == 0).all()) and not bool((k[~empty] == 0).all(-1).any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("q_len", [1, 6, 90])
def test_holes_are_not_seen(way, dtype, q_len):
    """Pages that a window has left behind may be taken away: their table entries are holes, and nothing of them is read."""
    s = Setup([q_len], [400], 2, 64, dtype, 16, seed=2)
    s.write_all()
    q = s.queries(4)
    want = s.cache.attention(q, s.batch, window=50, sinks=4)
    whole = s.table.clone()
    gone = range(1, (400 - q_len - 50) // 16)
    for p in gone:
        s.table[0, p] = -1 if p % 2 else 10 ** 6
    assert torch.equal(s.cache.attention(q, s.batch, window=50, sinks=4), want)
    # a hole inside what is seen counts as masked
    s.table.copy_(whole)
    s.table[0, 3] = -1
    s.table[0, 24] = -7 if q_len == 1 else s.table[0, 24]
    holes = [(0, 3)] + ([(0, 24)] if q_len == 1 else [])
    got, lse = s.cache.attention(q, s.batch, want_lse=True)
    check_attention(s, q, got, lse, exact_attention(s, q, holes=holes))
    # nothing but holes; nothing is written to a hole and zeros come back
    s.table.fill_(-1)
    got, lse = s.cache.attention(q, s.batch, want_lse=True)
    assert bool((got == 0).all()) and bool((lse == -math.inf).all())
    before = s.cache.k_pages.view(torch.uint8).clone()
    x = torch.ones(q_len, 2, 64, device=DEV)
    s.cache.write(x, x, s.batch)
    assert torch.equal(s.cache.k_pages.view(torch.uint8), before)
    assert bool((s.cache.read(s.batch)[0] == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("q_len,kv", [(1, 100), (8, 100), (70, 180), (150, 150)])
def test_what_is_masked_has_no_effect(way, dtype, bad, q_len, kv):
    """A later token's or a forgotten token's NaN or infinity does not reach the rows that do not see it; rows that see
    it are not finite where it is."""
    window, sinks, at, old = 40, 2, kv - 1, 7
    s = Setup([q_len], [kv], 2, 64, dtype, 16, seed=4)
    s.write_all()
    q = s.queries(6)
    clean = s.cache.attention(q, s.batch, window=window, sinks=sinks)
    n = sum(s.kv_lens)
    k = torch.cat([t.float() for t in s.k]); v = torch.cat([t.float() for t in s.v])
    for p in (at, old):
        k[p, 0, 3] = bad
        v[p, :, 10] = bad
    s.write_all(k=k, v=v)
    got = s.cache.attention(q, s.batch, window=window, sinks=sinks)
    pos = torch.arange(kv - q_len, kv, device=DEV)
    sees = (pos == at) | ((pos >= old) & (pos - old < window))
    assert torch.equal(got[~sees], clean[~sees])
    assert not bool(torch.isfinite(got[sees][:, :, 10]).any())
    assert bool(torch.isfinite(got[sees][:, 3:, :10]).all())                   # the other KV head's keys are as they were


@pytest.mark.parametrize("dtype", TYPES)
def test_nothing_but_nan_is_nan(way, dtype):
    s = Setup([1, 1], [50, 70], 1, 64, dtype)
    s.write_all()
    q = s.queries(2)
    q[0, 0, 0] = math.nan
    got, lse = s.cache.attention(q, s.batch, want_lse=True)
    assert bool(torch.isnan(got[0, 0]).all()) and bool(torch.isnan(lse[0, 0]))
    assert bool(torch.isfinite(got[0, 1]).all()) and bool(torch.isfinite(got[1]).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_large_scores(way, dtype):
    """Scores of hundreds: the running maximum keeps exponentials finite, in any order of the keys."""
    s = Setup([1, 20], [900, 900], 1, 64, dtype, seed=9)
    s.write_all()
    q = s.queries(4, 60.0)
    got, lse = s.cache.attention(q, s.batch, want_lse=True)
    out, z, mass = exact_attention(s, q)
    # scores of some hundreds are rounded at 2^-24 of that: probabilities are off by up to 1e-4, and so are outputs
    assert float((got.double() - out).abs().max()) <= (4e-4 if dtype == torch.float32 else 2e-2)
    assert float((lse.double() - z).abs().max()) <= 2e-6 * float(z.abs().max())


@pytest.mark.parametrize("dtype", TYPES)
def test_shared_pages_and_pieces(way, dtype):
    """Two sequences that share their first pages; a prompt taken in one call and in pieces gives the same rows."""
    s = Setup([96], [96], 2, 64, dtype, 16, seed=6)
    s.write_all()
    q = s.queries(4)
    whole = s.cache.attention(q, s.batch)
    table = torch.cat([s.table[:1], s.table[:1]])
    b = ead.PagedBatch.of(table, [10, 1], [96, 80])
    got = s.cache.attention(torch.cat([q[86:], q[79:80]]), b)
    tol = 2e-6 if dtype == torch.float32 else 2.0 ** -7
    assert float((got[:10].double() - whole[86:].double()).abs().max()) <= tol
    assert float((got[10].double() - whole[79].double()).abs().max()) <= tol


def test_a_long_sequence_in_a_large_pool(way):
    """Element offsets beyond 2^31: the last pages of a pool of 2.2e9 elements."""
    n_kv, hd, page = 8, 128, 256
    n_pages = (2 ** 31 + 2 ** 27) // (n_kv * hd * page)
    cache = ead.PagedCache.empty(n_pages, page, n_kv, hd, F8, DEV)
    g = torch.Generator(device=DEV); g.manual_seed(1)
    kv = 6000
    per = -(-kv // page)
    table = torch.arange(n_pages - per, n_pages, dtype=torch.int32, device=DEV)[None].contiguous()
    k, v = (torch.randn(kv, n_kv, hd, generator=g, device=DEV).bfloat16() for _ in range(2))
    cache.write(k, v, ead.PagedBatch.of(table, [kv], [kv]))
    rk, rv = cache.read(ead.PagedBatch.of(table, [kv], [kv]))
    assert torch.equal(rk.double(), exact_round(k, F8)[0]) and torch.equal(rv.double(), exact_round(v, F8)[0])
    for ql in (1, 100):
        q = torch.randn(ql, 16, hd, generator=g, device=DEV).bfloat16()
        got, lse = cache.attention(q, ead.PagedBatch.of(table, [ql], [kv]), want_lse=True)

        class s:  # noqa: N801
            q_lens, kv_lens = [ql], [kv]
        s.n_kv, s.hd, s.page, s.k, s.v = n_kv, hd, page, [rk.double()], [rv.double()]
        check_attention(s, q, got, lse, exact_attention(s, q))


@pytest.mark.parametrize("dtype", TYPES)
def test_a_graph_follows_its_lengths(way, dtype):
    """A captured step (write and attention) replayed while the lengths on the device grow, against eager calls."""
    n_kv, hd, steps = 2, 64, 5
    s = Setup([1, 1], [300, 1500], n_kv, hd, dtype, 16, seed=8, stale=0.0)
    s.write_all()
    lens = torch.tensor([290, 1490], dtype=torch.int32, device=DEV)
    starts = torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV)
    batch = ead.PagedBatch(s.table, starts, lens, rows=2, max_q=1, min_q=1, max_kv=1500)
    t = torch.float32 if dtype == torch.float32 else torch.bfloat16
    q, k, v = (torch.zeros(2, n, hd, device=DEV, dtype=t) for n in (6, n_kv, n_kv))
    out = torch.zeros_like(q)
    s.cache.write(k, v, batch); s.cache.attention(q, batch, out=out)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        s.cache.attention(q, batch, out=out)          # this stream's workspace
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s.cache.write(k, v, batch)
        s.cache.attention(q, batch, out=out)
        lens.add_(1)
    for step in range(steps):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=s.g, device=DEV))
        now = lens.tolist()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        again = ead.PagedBatch(s.table, starts, torch.tensor(now, dtype=torch.int32, device=DEV), rows=2, max_q=1, min_q=1, max_kv=1500)
        assert torch.equal(got, s.cache.attention(q, again))
        rk, _ = s.cache.read(again, torch.float32)
        assert torch.equal(rk.double(), exact_round(k, dtype)[0])
        assert lens.tolist() == [n + 1 for n in now]


def test_two_streams_have_their_own_workspaces(way):
    s = Setup([1], [6000], 1, 128, torch.bfloat16, 16)
    s.write_all()
    q = s.queries(8)
    want = s.cache.attention(q, s.batch)
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    outs = []
    for _ in range(20):
        for st in (a, b):
            with torch.cuda.stream(st):
                outs.append(s.cache.attention(q, s.batch))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_repeated_calls_are_bit_equal(way):
    s = Setup([1, 1, 30], [3000, 77, 900], 2, 128, F8, 32)
    s.write_all()
    q = s.queries(10)
    want = s.cache.attention(q, s.batch, want_lse=True)
    for _ in range(10):
        got = s.cache.attention(q, s.batch, want_lse=True)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_bounds_that_are_too_small_stay_in_range(way):
    """max_kv and max_q below what the device arrays say: reads and writes stay inside, rows up to max_q are right."""
    s = Setup([1, 1], [900, 500], 2, 64, torch.bfloat16, 16)
    s.write_all()
    q = s.queries(4)
    small = ead.PagedBatch(s.table, s.batch.q_starts, s.batch.kv_lens, rows=2, max_q=1, min_q=0, max_kv=10)
    assert float((s.cache.attention(q, small).float() - s.cache.attention(q, s.batch).float()).abs().max()) < 2.0 ** -7
    wild = ead.PagedBatch(s.table, torch.tensor([-5, 1, 999], dtype=torch.int32, device=DEV),
                          torch.tensor([10 ** 9, -3], dtype=torch.int32, device=DEV), rows=2, max_q=1, max_kv=900)
    s.cache.attention(q, wild)
    s.cache.read(wild)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch", [64, 65, 150, 1100])
def test_many_sequences(way, dtype, batch):
    """More sequences than a wave has lanes, and more than are cut into shares; some without rows, some with many."""
    rng = np.random.default_rng(batch)
    q_lens = rng.choice([0, 1, 1, 1, 2, 9], batch).tolist()
    kv_lens = [int(n) + q for n, q in zip(rng.integers(0, 1500 if batch < 1000 else 60, batch), q_lens)]
    s = Setup(q_lens, kv_lens, 2, 32, dtype, 16, seed=batch)
    s.write_all()
    q = s.queries(14, 1.5)
    got, lse = s.cache.attention(q, s.batch, want_lse=True)
    check_attention(s, q, got, lse, exact_attention(s, q))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads", [(8, 1, 32), (10, 2, 128)])
@pytest.mark.parametrize("window,sinks", [(17, 3), (129, 0), (70, 40)])
def test_windows_of_other_heads(way, dtype, heads, window, sinks):
    n_heads, n_kv, hd = heads
    s = Setup([1, 200, 33], [300, 333, 40], n_kv, hd, dtype, 64, seed=window)
    s.write_all()
    q = s.queries(n_heads, 1.5)
    got, lse = s.cache.attention(q, s.batch, window=window, sinks=sinks, want_lse=True)
    check_attention(s, q, got, lse, exact_attention(s, q, window, sinks))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k_scale,v_scale", [(2.0 ** 40, 2.0 ** -40), (2.0 ** -60, 2.0 ** 60)])
def test_magnitudes_far_from_one(way, dtype, k_scale, v_scale):
    """Powers of two in K, undone in the queries, and in V: the same attention, times V's."""
    s = Setup([1, 50], [200, 170], 2, 64, dtype, seed=3)
    n = sum(s.kv_lens)
    k, v = (torch.randn(n, 2, 64, generator=s.g, device=DEV) for _ in range(2))
    s.write_all(k=k, v=v)
    q = s.queries(6)
    want = s.cache.attention(q, s.batch)
    s.write_all(k=k * k_scale, v=v * v_scale)
    got = s.cache.attention((q.float() / k_scale).to(q.dtype), s.batch)
    assert torch.equal(got.double() / v_scale, want.double())


@pytest.mark.parametrize("dtype", [torch.bfloat16, F8])
@pytest.mark.parametrize("heads", [(8, 2, 64), (4, 4, 32), (4, 1, 128)])
def test_many_rows_over_long_contexts(dtype, heads):
    """More than 4096 keys: one bf16 term of each probability away from the edges.  A term is off by at most 2^-8 of itself (8 significant
    bits), and so is the output's rounding: 1.05 * 2^-8 (|out| + sum_j p_j |v_j|) + 1e-5."""
    n_heads, n_kv, hd = heads
    s = Setup([700, 450], [5000, 4700], n_kv, hd, dtype, 64, seed=1)
    s.write_all()
    q = s.queries(n_heads, 1.5)
    L = ead.lib()
    L.ead_test_paged.argtypes = [C.c_double, C.c_int32]
    L.ead_test_paged(0.0, 0)
    try:
        got, lse = s.cache.attention(q, s.batch, want_lse=True)
    finally:
        L.ead_test_paged(-1.0, 0)
    out, z, mass = exact_attention(s, q)
    bound = 1.05 * 2.0 ** -8 * (out.abs() + mass) + 1e-5
    assert bool(((got.double() - out).abs() <= bound).all())
    assert float((lse.double() - z).abs().max()) <= 1e-5


def test_refusals():
    s = Setup([2, 1], [20, 5], 2, 64, torch.bfloat16, 16)
    s.write_all()
    q = s.queries(4)
    k = torch.zeros(3, 2, 64, device=DEV, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        s.cache.attention(q[:2], s.batch)                                  # rows
    with pytest.raises(ValueError):
        s.cache.attention(q.float(), s.batch)                              # type
    with pytest.raises(TypeError):
        s.cache.attention(q.half(), s.batch)
    with pytest.raises(ead.EadError):
        s.cache.attention(torch.zeros(3, 3, 64, device=DEV, dtype=torch.bfloat16), s.batch)    # 3 heads over 2
    with pytest.raises(ead.EadError):
        s.cache.attention(q, s.batch, window=-1)
    with pytest.raises(ead.EadError):
        s.cache.attention(q, s.batch, scale=0.0)
    with pytest.raises(ead.EadError):
        s.cache.attention(q, s.batch, scale=math.nan)
    with pytest.raises(ValueError):
        s.cache.write(k, k.float(), s.batch)
    with pytest.raises(ValueError):
        s.cache.write(k.transpose(0, 2).contiguous().transpose(0, 2), k, s.batch)
    with pytest.raises(ValueError):
        s.cache.write(k.cpu(), k, s.batch)
    with pytest.raises(ValueError):
        ead.PagedCache(s.cache.k_pages.view(F8), s.cache.v_pages.view(F8))
    with pytest.raises(ValueError):
        ead.PagedCache(s.cache.k_pages[:, :, ::2], s.cache.v_pages[:, :, ::2])
    odd = ead.PagedCache.empty(4, 24, 2, 64, torch.bfloat16, DEV)
    with pytest.raises(ead.EadError):
        odd.write(k, k, s.batch)                                           # page size
    with pytest.raises(ead.EadError):
        ead.PagedCache.empty(4, 16, 2, 48, torch.bfloat16, DEV).write(k[..., :48], k[..., :48], s.batch)
    with pytest.raises(ValueError):
        ead.PagedBatch(s.table.long(), s.batch.q_starts, s.batch.kv_lens, rows=3, max_q=2, max_kv=20)
    with pytest.raises(ValueError):
        ead.PagedBatch(s.table, s.batch.q_starts[:-1], s.batch.kv_lens, rows=3, max_q=2, max_kv=20)
    with pytest.raises(ValueError):
        ead.PagedBatch.of(s.table, [1, -1], [2, 2])
    none = ead.PagedBatch.of(s.table, [0, 0], [20, 5])                     # a step without rows is none
    assert s.cache.attention(q[:0], none).shape == (0, 4, 64) and s.cache.read(none)[0].shape == (0, 2, 64)
    s.cache.write(k[:0], k[:0], none)
