"""Log probabilities, ranks, entropies and the most likely tokens against their definitions in 64 bits.

Tolerances.  Tokens and ranks are compared exactly.  With d = (l - m) log2 e, u = 2^-24 and n additions in a lane's sum (a row's logits over at least 256 lanes, plus
the joins): every 2^d is off by u |d| ln 2 + 2u of itself, the sum by n u more, so ln Z is off by (n + 2) u + u E|d|, and a log probability by that and the
rounding of d and of the result.  The entropy is ln Z + E[m - l]: its second part is off by the same share of E|d|."""
import ctypes as C
import math

import pytest
import torch

import paper_2502_06833_amd as ead

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


def exact(x, tokens, top):
    """Row by row in 64 bits; NaN where there is no distribution."""
    x = x.double()
    rank = torch.where(torch.isnan(x), -math.inf, x)
    bad = torch.isnan(x).any(1) | (x == math.inf).any(1) | (rank.amax(1) == -math.inf)
    m = rank.amax(1, keepdim=True)
    m = torch.where(torch.isfinite(m), m, 0.0)
    d = rank - m
    p = d.exp()
    z = p.sum(1)
    far = torch.where(p > 0, -d, 0.0)
    h = z.log() + (p * far).sum(1) / z
    lp = d - z.log()[:, None]
    h[bad], lp[bad] = math.nan, math.nan
    out = {"H": h, "far": (p * far).sum(1) / z, "order": torch.sort(rank, dim=1, descending=True, stable=True).indices[:, :top]}
    out["top"] = lp.gather(1, out["order"])
    if tokens is not None:
        ok = (tokens >= 0) & (tokens < x.shape[1])
        t = tokens.long().clamp(0, x.shape[1] - 1)[:, None]
        out["lp"] = torch.where(ok, lp.gather(1, t)[:, 0], 0.0)
        out["rank"] = torch.where(ok, (x > x.gather(1, t)).sum(1) + 1, 0)
    return out


def near(got, want, tol):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), (got, want)
    assert torch.equal(torch.isinf(got), torch.isinf(want)) and torch.equal(got[torch.isinf(want)], want[torch.isinf(want)])
    f = torch.isfinite(want)
    over = ((got - want).abs() - tol.expand_as(want))[f]
    assert over.numel() == 0 or float(over.max()) <= 0, float(over.max())


def check(x, r, tokens, top, unit=ead.NATS):
    want = exact(x, tokens, top)
    n = x.shape[1] / 256 + 80
    far = torch.nan_to_num(want["far"])
    tol = U * (n + 4 + 2 * far)
    per = 1 / math.log(2) if unit == ead.BITS else 1.0
    near(r.H, want["H"] * per, per * (tol * (1 + far) + 4 * U * torch.nan_to_num(want["H"]).abs()))
    if tokens is not None:
        near(r.logprob, want["lp"], tol + 4 * U * torch.nan_to_num(want["lp"], neginf=0.0).abs())
        assert torch.equal(r.rank.long(), want["rank"])
    if top:
        assert torch.equal(r.top_tokens.long(), want["order"])
        near(r.top_logprobs, want["top"], tol[:, None] + 4 * U * torch.nan_to_num(want["top"], neginf=0.0).abs())


def rows(n, vocab, dtype, seed=0, scale=2.0):
    g = torch.Generator(device=DEV); g.manual_seed(seed)
    x = (scale * torch.randn(n, vocab, generator=g, device=DEV)).to(dtype)
    t = torch.randint(vocab, (n,), generator=g, device=DEV).to(torch.int32)
    return x, t


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,vocab", [(1, 1), (3, 2), (2, 7), (5, 33), (1, 2047), (4, 2048), (3, 2049), (2, 4099), (1, 50257), (3, 151936), (700, 1000), (1100, 333), (513, 8200)])
@pytest.mark.parametrize("top", [0, 1, 5, 32])
def test_shapes(dtype, n, vocab, top):
    top = min(top, vocab)
    x, t = rows(n, vocab, dtype, seed=n + vocab)
    check(x, ead.logprobs(x, t, top=top), t, top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("first,wide", [(0, 1), (1, 0), (3, 4), (5, 9), (8, 8)])
def test_strides_and_alignments(dtype, first, wide):
    """Rows inside a wider tensor, at starts that are and are not 16-byte boundaries; what lies around them is NaN."""
    vocab, n = 5001, 9
    big = torch.full((n, first + vocab + wide), math.nan, device=DEV, dtype=dtype)
    x, t = rows(n, vocab, dtype, seed=first)
    view = big[:, first:first + vocab]
    view.copy_(x)
    check(x, ead.logprobs(view, t, top=20), t, 20)
    one = ead.logprobs(x[:1].expand(4, -1), t[:1].expand(4).contiguous(), top=3)             # the same row four times
    check(x[:1].expand(4, -1), one, t[:1].expand(4), 3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masks(dtype):
    """-inf and the type's lowest value as masks, rows with fewer logits than alternatives, and rows with none."""
    vocab = 20011
    x, t = rows(12, vocab, dtype, seed=3)
    low = torch.finfo(dtype).min
    keep = torch.zeros(vocab, dtype=torch.bool, device=DEV)
    keep[[5, 77, 4096, 4097, 20010]] = True
    x[0][~keep] = -math.inf
    x[1][~keep] = low
    x[2] = -math.inf
    x[3] = low
    x[4] = -math.inf
    x[4, 20000] = -300.0
    x[5] = -math.inf
    x[5, 0] = low
    x[6, :20000] = -math.inf
    x[7, 3:] = low
    t[0], t[1], t[2], t[4], t[6], t[8], t[9] = 77, 6, 1, 20000, 4, -1, vocab
    r = ead.logprobs(x, t, top=20)
    check(x, r, t, 20)
    assert float(r.logprob[6]) == -math.inf and float(r.logprob[8]) == 0 and int(r.rank[8]) == 0 and int(r.rank[9]) == 0
    assert abs(float(r.H[3]) - math.log(vocab)) < 1e-4 and float(r.H[4]) == 0 and math.isnan(float(r.H[2]))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_numbers_that_are_none(dtype):
    vocab = 9001
    x, t = rows(6, vocab, dtype, seed=4)
    x[0, 17], x[1, 9000], x[2, 4], x[3] = math.nan, math.inf, math.inf, math.nan
    x[2, 5] = math.inf
    x[4, 0], t[4] = math.nan, 0
    t[1] = 3
    r = ead.logprobs(x, t, top=7)
    check(x, r, t, 7)
    assert r.top_tokens[2, :2].tolist() == [4, 5] and r.top_tokens[3].tolist() == list(range(7)) and math.isfinite(float(r.H[5]))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("top", [1, 20, 32])
def test_ties_and_orders(dtype, top):
    vocab = 30011
    at = torch.arange(vocab, device=DEV)
    x = torch.stack([torch.zeros(vocab, device=DEV), at / 256.0, -at / 256.0, (at * 7919 % 13).float(), (at % 2).float(), torch.where(at % 2 == 0, 0.0, -0.0),
                     torch.where(at > 29000, 3.0, 0.0), torch.where(at % 64 < 20, 5.0 + at / 8192, 0.0)]).to(dtype)
    t = torch.tensor([0, 30010, 17, 13, 1, 8, 5, 19], dtype=torch.int32, device=DEV)
    check(x, ead.logprobs(x, t, top=top), t, top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", [1e4, -1e4, 1e20, 3e37, -2e38, 3e38])
def test_large_logits(dtype, shift):
    """Differences of logits are what counts, however large they are themselves (their own rounding to the type comes first)."""
    x, t = rows(4, 6007, dtype, seed=5)
    x = (x.float() * max(1.0, abs(shift) * 2.0 ** -9) + shift).clamp(torch.finfo(dtype).min, torch.finfo(dtype).max).to(dtype)
    check(x, ead.logprobs(x, t, top=5), t, 5)


def test_entropy_is_that_of_entropy_argmax():
    for dtype in (torch.float32, torch.bfloat16):
        x, t = rows(33, 50264, dtype, seed=6)
        for unit in (ead.NATS, ead.BITS):
            r = ead.logprobs(x, t, top=1, unit=unit)
            check(x, r, t, 1, unit)
            h, a = ead.entropy_argmax(x, unit=unit)
            assert torch.equal(a, r.top_tokens[:, 0]) and float((h - r.H).abs().max()) < 1e-4


def test_nothing_but_what_is_asked_for():
    x, t = rows(3, 4000, torch.bfloat16)
    r = ead.logprobs(x)
    assert r.logprob is None and r.rank is None and r.top_tokens is None
    check(x, r, None, 0)
    assert ead.logprobs(x[:0], t[:0], top=4).top_tokens.shape == (0, 4)


def test_the_same_every_time():
    x, t = rows(5, 151936, torch.bfloat16, seed=7)
    first = ead.logprobs(x, t, top=20)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, ead.logprobs(x, t, top=20)))


def test_calls_of_different_shapes_share_a_workspace():
    cases = [(1, 151936, 20), (64, 151936, 5), (7, 9000, 0), (300, 40000, 32), (1, 151936, 20), (900, 20000, 3)]
    data = [rows(n, v, torch.bfloat16, seed=i) for i, (n, v, _) in enumerate(cases)]
    for _ in range(2):
        for (x, t), (_, _, top) in zip(data, cases):
            check(x, ead.logprobs(x, t, top=top), t, top)


def test_streams_at_once():
    data = [rows(9, 100003, torch.float32, seed=i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in data]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(ead.logprobs(data[i][0], data[i][1], top=8))
    torch.cuda.synchronize()
    for i, (x, t) in enumerate(data):
        for r in got[i]:
            check(x, r, t, 8)


def test_captured_calls():
    """Two graphs, one captured before any eager call of the shape, replayed between eager calls and beside each other, on new logits every time."""
    xs = [rows(n, 70001, torch.bfloat16, seed=n) for n in (1, 40)]
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in xs]
    for x, t in xs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append((ead.logprobs(x, t, top=6), ead.logprobs(x, t, top=2)))
        graphs.append(g)
    for i in range(4):
        for j, (x, t) in enumerate(xs):
            x.copy_(rows(x.shape[0], x.shape[1], x.dtype, seed=100 * i + j)[0])
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        eager = [ead.logprobs(x, t, top=6) for x, t in xs]
        torch.cuda.synchronize()
        for (x, t), (six, two), e in zip(xs, outs, eager):
            assert all(torch.equal(a, b) for a, b in zip(six, e)) and torch.equal(two.top_tokens, e.top_tokens[:, :2])
            check(x, e, t, 6)
