"""The steps beside attention of a program that keeps its own caches, each in its plain form and through its entry point.

Five kinds of calls:

  rotate    the queries and keys of some rows: every head's vector over its root mean square, times a gain, then turned by
            the row's position
  append    the same on the way to a paged cache: rotated queries come back, rotated keys and the values go to their
            places in the pages, rounded to the cache's type
  logprobs  from logits: the log probability and the rank of a given token, the entropy, the most likely tokens
  weigh     every cached position's share of the attention that the rows' queries pay, added to what it had before
  evict     a sequence that holds more than `keep` positions is cut to that many, for every KV head on its own: its first
            and its last positions stay, and of the others those with the largest weights

`append`, `weigh` and `evict` work on one description of a batch (`page_table`, `q_starts`, `kv_lens`: sequence b holds
`kv_lens[b]` positions, the last `q_starts[b + 1] - q_starts[b]` of which are the call's rows).  Head layouts are those of
the model pairs the benchmark names.
"""
import math

import torch

own = False

DEV = "cuda:0"

# query heads, KV heads, head_dim, rotary base, float32 model
_HEADS = {
    "tiny-s": (4, 4, 32, 1e4, True),
    "tiny-l": (8, 8, 32, 1e4, True),
    "llama-1b": (32, 8, 64, 5e5, False),
    "llama-8b": (32, 8, 128, 5e5, False),
    "qwen-0.5b": (14, 2, 64, 1e6, False),
    "qwen-1.5b": (12, 2, 128, 1e6, False),
    "qwen-14b": (40, 8, 128, 1e6, False),
}
_CACHE = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}
_ROWS = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2, "fp8": 1}
_EPS = 1e-6


# ----------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one token of an interactive request: nothing but latency
        dict(name="rotate_step_b1", kind="rotate", heads="qwen-14b", rows="bf16", n=1, far=4096, norm=True),
        # the prompts of a batch, Q and K as slices of one projection's output
        dict(name="rotate_prompts", kind="rotate", heads="llama-8b", rows="bf16", n=16381, far=131072, norm=True, fused=True),
        # the flagship batch's decode step: one row for each of 64 sequences, keys and values to an 8-bit cache
        dict(name="append_step_b64_fp8", kind="append", heads="qwen-14b", rows="bf16", cache="fp8", page=16, batch=64, q_lo=1, q_hi=1,
             kv_lo=128, kv_hi=8192, norm=True),
        # ragged prompts to a bf16 cache, without norms (a Llama layout has none)
        dict(name="append_prompts_bf16", kind="append", heads="llama-8b", rows="bf16", cache="bf16", page=64, batch=23, q_lo=301, q_hi=2047,
             kv_lo=0, kv_hi=0, norm=False, fused=True),
        # what a request gets back with its token: log probability, rank, entropy, five alternatives
        dict(name="logprobs_b1_top5", kind="logprobs", rows="bf16", n=1, vocab=128256, top=5),
        # a decode step of the flagship batch with twenty alternatives
        dict(name="logprobs_b64_top20", kind="logprobs", rows="bf16", n=64, vocab=151936, top=20),
        # a text is scored: float32 logits of an odd vocabulary, given tokens only
        dict(name="logprobs_score_f32", kind="logprobs", rows="f32", n=1023, vocab=50257, top=0),
        # one interactive sequence at some thousand positions
        dict(name="weigh_b1_bf16", kind="weigh", heads="llama-8b", cache="bf16", page=16, batch=1, q_lo=1, q_hi=1, kv_lo=8190, kv_hi=8190,
             window=0, sinks=0),
        # a decode step over long ragged contexts in 8 bits
        dict(name="weigh_b64_fp8", kind="weigh", heads="qwen-14b", cache="fp8", page=64, batch=64, q_lo=1, q_hi=1, kv_lo=1024, kv_hi=16384,
             window=0, sinks=0),
        # a piece of a long prompt over what is in the cache already: matrix products and exponentials
        dict(name="weigh_chunk_bf16", kind="weigh", heads="llama-8b", cache="bf16", page=64, batch=1, q_lo=2048, q_hi=2048, kv_lo=6145, kv_hi=6145,
             window=0, sinks=0),
        # decoding within a budget: 64 sequences are cut back after some tokens more than they may hold
        dict(name="evict_b64_budget_fp8", kind="evict", heads="qwen-14b", cache="fp8", page=16, batch=64, kv_lo=2049, kv_hi=2176, keep=2048, sinks=4,
             recent=256),
        # long prompts are cut to half once they have been read
        dict(name="evict_prompts_bf16", kind="evict", heads="llama-8b", cache="bf16", page=64, batch=3, kv_lo=24001, kv_hi=32768, keep=12289, sinks=16,
             recent=1023),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "append", "logprobs", "logprobs", "weigh", "weigh", "evict"])
    if kind == "logprobs":
        vocab = _logint(rng, 500, 160000)
        n = _logint(rng, 1, max(1, min(2048, 60_000_000 // vocab)))
        return dict(kind=kind, rows=rng.choice(["bf16", "bf16", "f32"]), n=n, vocab=vocab, top=rng.choice([0, 1, 3, 5, 8, 20, 32]),
                    wide=rng.choice([0, 0, 1, 8, 64]), masked=rng.choice([0, 0, 0, 0.5, 0.999]))
    heads = rng.choice(sorted(_HEADS))
    f32 = _HEADS[heads][4]
    case = dict(kind=kind, heads=heads)
    if kind in ("rotate", "append"):
        case.update(rows="f32" if f32 else rng.choice(["bf16", "bf16", "f32"]), norm=rng.random() < 0.7, pairs=rng.random() < 0.3,
                    part=rng.choice([1.0, 1.0, 1.0, 0.5]), fused=rng.random() < 0.5)
        if kind == "rotate":
            case.update(n=_logint(rng, 1, 12000), far=_logint(rng, 100, 1000000))
            return case
        case.update(cache=rng.choice(["f32", "bf16"] if f32 else ["bf16", "bf16", "fp8"]), page=rng.choice([16, 32, 64, 128, 256]))
        q_hi = _logint(rng, 1, 64 if case["cache"] == "fp8" else 4000)
        batch = _logint(rng, 1, max(1, min(128, (1000 if case["cache"] == "fp8" else 16000) // q_hi)))
        kv_hi = _logint(rng, 1, 8000)
        case.update(batch=batch, q_lo=max(1, q_hi // rng.randint(1, 7)), q_hi=q_hi, kv_lo=kv_hi // rng.randint(1, 5), kv_hi=kv_hi)
        return case
    case.update(cache="f32" if f32 else rng.choice(["bf16", "fp8"]), page=rng.choice([16, 32, 64, 128, 256]))
    if kind == "evict":
        kv_hi = _logint(rng, 40, 40000)
        keep = max(8, int(kv_hi * rng.choice([0.25, 0.5, 0.8, 0.95])))
        case.update(batch=_logint(rng, 1, max(1, min(64, 150000 // kv_hi))), kv_lo=max(1, int(kv_hi * rng.choice([0.3, 0.9, 1.0]))), kv_hi=kv_hi,
                    keep=keep, sinks=min(rng.choice([0, 1, 4, 16]), keep // 3), recent=int(keep * rng.choice([0, 0.03, 0.2, 0.6])))
        return case
    form = rng.choice(["decode", "decode", "few", "chunk", "mixed"])
    if form == "decode":
        kv_hi, q_hi = _logint(rng, 2, 40000), 1
        batch = _logint(rng, 1, max(1, min(128, 600000 // kv_hi)))
    elif form == "few":
        kv_hi, q_hi = _logint(rng, 2, 16000), rng.randint(2, 24)
        batch = _logint(rng, 1, max(1, min(96, 200000 // kv_hi)))
    else:
        kv_hi, q_hi = _logint(rng, 2, 6000), _logint(rng, 25, 1500)
        batch = _logint(rng, 1, max(1, min(24, 12_000_000 // (q_hi * (kv_hi + q_hi)))))
    case.update(batch=batch, q_lo=1 if form in ("few", "mixed") else max(1, q_hi // rng.randint(1, 4)), q_hi=q_hi,
                kv_lo=kv_hi // rng.randint(1, 6), kv_hi=kv_hi, window=0, sinks=0)
    if rng.random() < 0.35:
        case.update(window=_logint(rng, 1, 6000), sinks=rng.choice([0, 1, 4, 16, 33]))
    if form == "mixed":
        case["steps"] = rng.randint(0, batch)
    return case


def _lens(case):
    """New rows and held positions of each sequence: spread over the case's ranges, the first `steps` sequences with one row."""
    b = case["batch"]

    def spread(lo, hi, salt):
        return [lo + int((hi - lo + 1) * ((salt + 0.6180339887 * i) % 1.0)) for i in range(b)]

    before = spread(case["kv_lo"], case["kv_hi"], 0.37)
    if case["kind"] == "evict":
        return [0] * b, before
    q = spread(case["q_lo"], case["q_hi"], 0.9999)
    q = [1 if i < case.get("steps", 0) else n for i, n in enumerate(q)]
    return q, [n + m for n, m in zip(q, before)]


def _seen(q_len, kv_len, window, sinks):
    """(pairs of a row and a position it sees, positions that any row sees) of one sequence."""
    first = kv_len - q_len
    if not window:
        return q_len * first + q_len * (q_len + 1) // 2, kv_len
    los = [max(0, p - window + 1) for p in range(first, kv_len)]
    return sum(first + i + 1 - lo + min(sinks, lo) for i, lo in enumerate(los)), kv_len - los[0] + min(sinks, los[0])


def work(case):
    kind = case["kind"]
    if kind == "logprobs":
        cells = case["n"] * case["vocab"]
        return dict(bytes=cells * _BYTES[case["rows"]] + case["n"] * (16 + 8 * case["top"]), flops=6 * cells)
    n_heads, n_kv, hd = _HEADS[case["heads"]][:3]
    if kind == "rotate":
        cells = case["n"] * (n_heads + n_kv) * hd
        return dict(bytes=2 * cells * _BYTES[case["rows"]] + 4 * case["n"], flops=6 * cells)
    q, kv = _lens(case)
    rows = sum(q)
    held = n_kv * (hd * _BYTES[case["cache"]] + (1 if case["cache"] == "fp8" else 0))     # K or V of a position
    if kind == "append":
        esz = _BYTES[case["rows"]]
        return dict(bytes=rows * (2 * n_heads * hd * esz + 2 * n_kv * hd * esz + 2 * held), flops=6 * rows * (n_heads + n_kv) * hd)
    if kind == "weigh":
        esz = 4 if case["cache"] == "f32" else 2
        seen = [_seen(n, m, case["window"], case["sinks"]) for n, m in zip(q, kv)]
        return dict(bytes=sum(s for _, s in seen) * (held + 8 * n_kv) + rows * n_heads * (hd * esz + 4),
                    flops=(2 * hd + 3) * n_heads * sum(p for p, _ in seen))
    total = 0.0
    for n in kv:
        total += 4 * n_kv * case["keep"]                                                   # which position lies where now
        if n > case["keep"]:
            middle, stay = n - case["sinks"] - case["recent"], case["keep"] - case["sinks"] - case["recent"]
            moved = case["recent"] + (n - case["keep"]) * stay / middle                    # weights know nothing of places: those past the cut
            total += 4 * n_kv * middle + 2 * moved * (2 * held + 4 * n_kv)
    return dict(bytes=int(total), flops=0)


# ----------------------------------------------------------------------------------------- inputs
def _scale_of(exponents):
    """The powers of two that a cache in 8 bits keeps: 2^(e - 127), e >= 1."""
    return (exponents.to(torch.int32) << 23).view(torch.float32)


def _round_to_8(x):
    """e4m3 codes and exponents of vectors: the smallest power of two that brings the largest magnitude to 448 or less."""
    m, e = torch.frexp(x.abs().amax(-1))
    e = torch.where(m > 0, torch.where(m <= 0.875, e - 9, e - 8) + 127, torch.ones_like(e)).clamp(1, 254).to(torch.uint8)
    return (x / _scale_of(e)[..., None]).to(torch.float8_e4m3fn), e


def _prepare_logprobs(case, g):
    n, vocab, t = case["n"], case["vocab"], _ROWS[case["rows"]]
    # a few tokens stand out, most do not: normal logits, and some raised by what falls off like their rank
    x = 2.0 * torch.randn(n, vocab + case.get("wide", 0), generator=g, device=DEV)
    apart = vocab // 40
    hot = torch.randint(vocab, (n, 1), generator=g, device=DEV) + torch.randint(apart, (n, 40), generator=g, device=DEV)
    hot = (hot + apart * torch.arange(40, device=DEV)) % vocab                             # no token twice
    x.scatter_(1, hot, 12.0 - 2.0 * torch.arange(1, 41, device=DEV).log() + torch.randn(n, 40, generator=g, device=DEV))
    if case.get("masked"):                                     # a grammar leaves some tokens only
        x.masked_fill_(torch.rand(x.shape, generator=g, device=DEV) < case["masked"], -math.inf)
        x.scatter_(1, hot, torch.randn(n, 40, generator=g, device=DEV))
    x = x.to(t)[:, :vocab]
    tokens = torch.where(torch.rand(n, generator=g, device=DEV) < 0.7, hot[:, 0], torch.randint(vocab, (n,), generator=g, device=DEV))
    tokens[3::11] = -1                                         # rows that only fill a batch up
    return dict(case=case, logits=x, tokens=tokens.to(torch.int32))


def _prepare_rotary(s, g):
    """Gains and the plan that a program keeps for a model."""
    case = s["case"]
    hd, theta = _HEADS[case["heads"]][2:4]
    s["theta"], s["rotary"] = theta, int(hd * case.get("part", 1.0))
    s["gains"] = tuple(1.0 + 0.2 * torch.randn(hd, generator=g, device=DEV) if case["norm"] else None for _ in "qk")
    if own:
        import paper_2502_06833_amd as ead
        s["plan"] = ead.Rotary(hd, theta, rotary_dim=s["rotary"], interleaved=case.get("pairs", False), q_gain=s["gains"][0], k_gain=s["gains"][1], eps=_EPS)


def _prepare_rows(s, n, g):
    case = s["case"]
    n_heads, n_kv, hd = _HEADS[case["heads"]][:3]
    t = _ROWS[case["rows"]]
    if case.get("fused"):                                      # Q, K and V side by side, as one projection leaves them
        qkv = (1.7 * torch.randn(n, n_heads + 2 * n_kv, hd, generator=g, device=DEV)).to(t)
        s["q"], s["k"], s["v"] = qkv[:, :n_heads], qkv[:, n_heads:n_heads + n_kv], qkv[:, n_heads + n_kv:]
    else:
        s["q"], s["k"], s["v"] = ((1.7 * torch.randn(n, h, hd, generator=g, device=DEV)).to(t) for h in (n_heads, n_kv, n_kv))


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1000003 + 7)
    kind = case["kind"]
    if kind == "logprobs":
        return _prepare_logprobs(case, g)
    n_heads, n_kv, hd = _HEADS[case["heads"]][:3]
    s = dict(case=case)
    if kind == "rotate":
        _prepare_rotary(s, g)
        _prepare_rows(s, case["n"], g)
        s["positions"] = torch.randint(case["far"], (case["n"],), generator=g, device=DEV).to(torch.int32)
        return s
    q_lens, kv_lens = _lens(case)
    ps, rows = case["page"], sum(q_lens)
    per = [-(-n // ps) for n in kv_lens]
    n_pages, wide = sum(per) + 5, max(per) + 2
    places = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    at = torch.arange(wide, device=DEV)
    counts = torch.tensor(per, device=DEV)
    index = (counts.cumsum(0) - counts)[:, None] + at
    table = torch.where(at < counts[:, None], places[index.clamp(max=n_pages - 1)], places[n_pages - 1]).to(torch.int32).contiguous()
    s.update(table=table, q_starts=torch.tensor([0] + q_lens, device=DEV).cumsum(0).to(torch.int32), rows=rows, max_q=max(q_lens), min_q=min(q_lens),
             kv_lens=torch.tensor(kv_lens, device=DEV, dtype=torch.int32), max_kv=max(kv_lens))
    # some channels of K are several times the others, as rotary keys have them
    loud = torch.where(torch.rand(n_kv, 1, hd, generator=g, device=DEV) < 0.06, 3.0, 0.9)

    def pages(channels):
        x = torch.randn(n_pages, n_kv, ps, hd, generator=g, device=DEV)
        x *= channels
        if case["cache"] == "fp8":
            return _round_to_8(x)
        return x.to(_CACHE[case["cache"]]), None

    s["k_pages"], s["k_scales"] = pages(loud)
    s["v_pages"], s["v_scales"] = pages(torch.ones_like(loud))
    if kind == "append":
        _prepare_rotary(s, g)
        _prepare_rows(s, rows, g)
    else:
        # what the positions have had so far: a few much, most little, some nothing at all
        w = torch.exp(torch.randn(n_pages, n_kv, ps, generator=g, device=DEV))
        w *= n_heads / n_kv / s["max_kv"]                      # as after some steps
        s["weights"] = w.masked_fill_(torch.rand(w.shape, generator=g, device=DEV) < 0.05, 0.0)
    if kind == "weigh":
        t = torch.float32 if case["cache"] == "f32" else torch.bfloat16
        s["q"] = (1.5 * torch.randn(rows, n_heads, hd, generator=g, device=DEV)).to(t)
        # the logarithms of the rows' sums as attention returns them, for normal keys of those channels
        seq, pos = _row_places(s)
        seen = pos + 1
        if case["window"]:
            seen = torch.where(pos >= case["window"], (case["window"] + (pos - case["window"] + 1).clamp(max=case["sinks"])), seen)
        var = (s["q"].float().view(rows, n_kv, -1, hd) * loud).square().sum(-1).view(rows, n_heads) / hd
        s["lse"] = torch.log(seen.float())[:, None] + var / 2
    if kind == "evict":
        s["scores"] = s["weights"].clone()                     # what is chosen by; the weights move with their positions
    if own:
        import paper_2502_06833_amd as ead
        s["cache"] = ead.PagedCache(s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"])
        s["batch"] = ead.PagedBatch(table, s["q_starts"], s["kv_lens"], rows=rows, max_q=s["max_q"], min_q=s["min_q"], max_kv=s["max_kv"])
    return s


# ----------------------------------------------------------------------------------------- the plain forms
def _row_places(s):
    """Sequence and position of every row."""
    row = torch.arange(s["rows"], device=DEV)
    seq = torch.searchsorted(s["q_starts"][1:].contiguous(), row, right=True)
    return seq, s["kv_lens"][seq] - s["q_starts"][seq + 1] + row


def _turned(s, x, gain, positions):
    """Float32 vectors, over their root mean square and times the gain where there is one, turned by their positions."""
    x = x.float()
    if gain is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS) * gain
    half = s["rotary"] // 2
    angle = positions.double()[:, None, None] * s["theta"] ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
    cos, sin = angle.cos().float(), angle.sin().float()
    turn, rest = x[..., :2 * half], x[..., 2 * half:]
    if s["case"].get("pairs"):
        a, b = turn[..., 0::2], turn[..., 1::2]
        turn = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = turn[..., :half], turn[..., half:]
        turn = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turn, rest], -1)


def _put(x, pages, scales, page, slot):
    if scales is None:
        pages[page, :, slot] = x.to(pages.dtype)
    else:
        codes, e = _round_to_8(x)
        pages.view(torch.uint8)[page, :, slot] = codes.view(torch.uint8)
        scales[page, :, slot] = e


def _pages_of(s, *more):
    return {n: s[n] for n in ("k_pages", "v_pages", "k_scales", "v_scales") + more if s[n] is not None}


def _plain_rotate(s):
    return tuple(_turned(s, s[n], gain, s["positions"]).to(s[n].dtype) for n, gain in zip("qk", s["gains"]))


def _plain_append(s):
    seq, pos = _row_places(s)
    ps = s["case"]["page"]
    page, slot = s["table"][seq, pos // ps].long(), pos % ps
    _put(_turned(s, s["k"], s["gains"][1], pos), s["k_pages"], s["k_scales"], page, slot)
    _put(s["v"].float(), s["v_pages"], s["v_scales"], page, slot)
    return {"q": _turned(s, s["q"], s["gains"][0], pos).to(s["q"].dtype), **_pages_of(s)}


def _ranked(x):
    """Whole numbers in the order of float32 values, the largest largest (-0 as 0)."""
    i = (x + 0.0).view(torch.int32).long()
    return torch.where(i < 0, -(i & 0x7FFFFFFF), i)


def _plain_logprobs(s):
    case, t = s["case"], s["tokens"].long()
    x = s["logits"].float()
    d = x - x.amax(-1, keepdim=True)
    p = d.exp()
    z = p.sum(-1)
    out = {"H": z.log() - (p * d.masked_fill(p == 0, 0.0)).sum(-1) / z}
    given = t >= 0
    mine = x.gather(1, t.clamp(min=0)[:, None])
    out["logprob"] = torch.where(given, d.gather(1, t.clamp(min=0)[:, None])[:, 0] - z.log(), 0.0)
    out["rank"] = torch.where(given, (x > mine).sum(-1) + 1, 0).to(torch.int32)
    if case["top"]:
        # equal logits: the lower token first
        key = (_ranked(x) << 20) + (0xFFFFF - torch.arange(case["vocab"], device=DEV))
        top = torch.topk(key, case["top"], -1).indices
        out["top_tokens"], out["top_logprobs"] = top.to(torch.int32), d.gather(1, top) - z.log()[:, None]
    return out


def _plain_weigh(s):
    case, q, ps = s["case"], s["q"], s["case"]["page"]
    n_heads, n_kv, hd = _HEADS[case["heads"]][:3]
    batch, group, max_q, per = case["batch"], n_heads // n_kv, s["max_q"], -(-s["max_kv"] // ps)
    ids = s["table"][:, :per].long()
    if s["k_scales"] is None:
        k = s["k_pages"][ids].float()
    else:
        k = s["k_pages"].view(torch.uint8)[ids].view(torch.float8_e4m3fn).float() * _scale_of(s["k_scales"][ids])[..., None]
    k = k.transpose(1, 2).reshape(batch, n_kv, -1, hd)
    starts = s["q_starts"][:-1].long()
    q_lens = s["q_starts"][1:] - s["q_starts"][:-1]
    at = torch.arange(max_q, device=DEV)
    rows = (starts[:, None] + at).clamp(max=s["rows"] - 1)
    held = torch.arange(per * ps, device=DEV)
    x = q[rows].float().view(batch, max_q, n_kv, group, hd).permute(0, 2, 1, 3, 4).reshape(batch, n_kv, max_q * group, hd)
    scores = torch.matmul(x, k.transpose(2, 3)).mul_(hd ** -0.5).view(batch, n_kv, max_q, group, -1)
    scores.sub_(s["lse"][rows].view(batch, max_q, n_kv, group).transpose(1, 2)[..., None])
    first = s["kv_lens"] - q_lens
    pos = (first[:, None] + at)[..., None]
    seen = (held <= pos) & (at < q_lens[:, None])[..., None]
    if case["window"]:
        seen &= (held > pos - case["window"]) | (held < case["sinks"])
    paid = scores.exp_().masked_fill_(~seen.view(batch, 1, max_q, 1, -1), 0.0).sum((2, 3))
    before = s["weights"][ids].transpose(1, 2).reshape(batch, n_kv, -1)
    new = paid + torch.where(held < first[:, None], before.transpose(0, 1), 0.0).transpose(0, 1)     # the rows' own positions had nothing yet
    new = torch.where((held < s["kv_lens"][:, None])[:, None], new, before)
    s["weights"][ids] = new.view(batch, n_kv, per, ps).transpose(1, 2)
    return s["weights"]


def _plain_evict(s):
    case, ps = s["case"], s["case"]["page"]
    n_kv = _HEADS[case["heads"]][1]
    batch, keep, sinks, recent, per = case["batch"], case["keep"], case["sinks"], case["recent"], -(-s["max_kv"] // ps)
    stay, cut = keep - sinks - recent, keep - recent
    ids = s["table"][:, :per].long()
    at = torch.arange(per * ps, device=DEV)
    lens = s["kv_lens"].long()[:, None, None]
    score = s["scores"][ids].transpose(1, 2).reshape(batch, n_kv, -1)
    # larger weights first, of equal ones the lower position; first and last positions are not asked
    key = (_ranked(score) << 20) + (0xFFFFF - at)
    key = torch.where((at >= sinks) & (at < lens - recent), key, -(1 << 62) - at)
    chosen = torch.zeros(key.shape, dtype=torch.bool, device=DEV)
    if stay and key.shape[-1] > stay:
        chosen.scatter_(-1, torch.topk(key, stay, -1).indices, True)
    chosen &= (at >= sinks) & (at < lens - recent)
    # the chosen ones past the cut go, in their order, to the places that others leave free
    free, moved = ~chosen & (at >= sinks) & (at < cut), chosen & (at >= cut)
    nth = lambda m: torch.where(m, m.cumsum(-1) - 1, per * ps)  # noqa: E731
    source = torch.zeros(batch, n_kv, per * ps + 1, dtype=torch.long, device=DEV)
    source.scatter_(-1, nth(moved), at.expand(batch, n_kv, -1))
    kept = torch.where(free, source.gather(-1, nth(free)), at)
    kept = torch.where((at >= cut) & (at < keep), lens - keep + at, kept)
    kept = torch.where(lens > keep, kept, at).expand(batch, n_kv, -1)
    kept = torch.where(at < lens.clamp(max=keep), kept, -1)[..., :keep]
    if kept.shape[-1] < keep:
        kept = torch.nn.functional.pad(kept, (0, keep - kept.shape[-1]), value=-1)
    live = kept >= 0
    seq = torch.arange(batch, device=DEV)[:, None, None].expand_as(kept)[live]
    head = torch.arange(n_kv, device=DEV)[None, :, None].expand_as(kept)[live]
    old, slot = kept[live], torch.arange(keep, device=DEV).expand_as(kept)[live]
    src, dst = (s["table"][seq, p // ps].long() for p in (old, slot))
    for pages in (s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"], s["weights"]):
        if pages is not None:
            pages = pages.view(torch.uint8) if pages.dtype == torch.float8_e4m3fn else pages
            pages[dst, head, slot % ps] = pages[src, head, old % ps]
    return {"kept": kept.to(torch.int32), **_pages_of(s, "weights")}


def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if not own:
        return {"rotate": _plain_rotate, "append": _plain_append, "logprobs": _plain_logprobs, "weigh": _plain_weigh, "evict": _plain_evict}[kind](s)
    if kind == "rotate":
        return s["plan"](s["q"], s["k"], s["positions"])
    if kind == "append":
        q = s["cache"].append(s["q"], s["k"], s["v"], s["batch"], s["plan"])
        return {"q": q, **_pages_of(s)}
    if kind == "logprobs":
        import paper_2502_06833_amd as ead
        r = ead.logprobs(s["logits"], s["tokens"], top=case["top"])
        out = {"H": r.H, "logprob": r.logprob, "rank": r.rank}
        if case["top"]:
            out.update(top_tokens=r.top_tokens, top_logprobs=r.top_logprobs)
        return out
    if kind == "weigh":
        s["cache"].weigh(s["q"], s["lse"], s["batch"], s["weights"], window=case["window"], sinks=case["sinks"])
        return s["weights"]
    kept = s["cache"].evict(s["batch"], s["scores"], case["keep"], sinks=case["sinks"], recent=case["recent"], weights=s["weights"])
    return {"kept": kept, **_pages_of(s, "weights")}


# ----------------------------------------------------------------------------------------- the definition, in 64 bits
def _exact_turned(s, x, gain, pos):
    """One row at a time of the definition: complex numbers times unit ones."""
    x = x.double()
    if gain is not None:
        x = x / torch.sqrt(torch.mean(x * x, -1, keepdim=True) + _EPS) * gain.double()
    r = s["rotary"]
    i = torch.arange(0, r, 2, device=DEV, dtype=torch.float64)
    unit = torch.polar(torch.ones(len(pos), r // 2, device=DEV, dtype=torch.float64), pos.double()[:, None] * torch.exp(-math.log(s["theta"]) * i / r))
    out = x.clone()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if s["case"].get("pairs") else (slice(0, r // 2), slice(r // 2, r))
    z = torch.complex(x[..., first], x[..., second]) * unit[:, None]
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _exact_append(s, q_lens, kv_lens):
    ps, row, qs, out = s["case"]["page"], 0, [], {n: s[n].double() for n in ("k_pages", "v_pages")}
    scales = {n: s[n].clone() for n in ("k_scales", "v_scales") if s[n] is not None}
    for b, (ql, kv) in enumerate(zip(q_lens, kv_lens)):
        part = slice(row, row + ql)
        row += ql
        pos = torch.arange(kv - ql, kv, device=DEV)
        qs.append(_exact_turned(s, s["q"][part], s["gains"][0], pos))
        page = s["table"][b].long()[pos // ps]
        for name, x in (("k", _exact_turned(s, s["k"][part], s["gains"][1], pos)), ("v", s["v"][part].double())):
            if scales:
                e = torch.ceil(torch.log2(x.abs().amax(2) / 448)).clamp(-126, 127)
                scales[name + "_scales"][page, :, pos % ps] = (e + 127).to(torch.uint8)
                x = x * torch.pow(torch.tensor(2.0, dtype=torch.float64, device=DEV), -e)[..., None]
            out[name + "_pages"][page, :, pos % ps] = x
    return {"q": torch.cat(qs), **out, **scales}


def _exact_logprobs(s):
    case = s["case"]
    lp, rank, h, top = [], [], [], []
    for x, t in zip(s["logits"], s["tokens"].tolist()):
        x = x.double()
        y = x - torch.logsumexp(x, 0)
        h.append(-(torch.exp(y) * torch.nan_to_num(y, neginf=0.0)).sum())
        lp.append(y[t] if t >= 0 else torch.zeros_like(h[-1]))
        if case["top"]:
            top.append(torch.sort(y, descending=True).values[:case["top"]])
    out = {"H": torch.stack(h), "logprob": torch.stack(lp), "rank": None}
    if case["top"]:
        out.update(top_tokens=None, top_logprobs=torch.stack(top))
    return out


def _exact_weigh(s, q_lens, kv_lens):
    case, ps, row = s["case"], s["case"]["page"], 0
    n_heads, n_kv, hd = _HEADS[case["heads"]][:3]
    out = s["weights"].double()
    for b, (ql, kv) in enumerate(zip(q_lens, kv_lens)):
        ids = s["table"][b, :-(-kv // ps)].long()
        k = s["k_pages"][ids.tolist()].double() if s["k_scales"] is None else torch.stack([s["k_pages"][i].double() for i in ids.tolist()])
        if s["k_scales"] is not None:
            k = k * torch.pow(torch.tensor(2.0, dtype=torch.float64, device=DEV), s["k_scales"][ids].double() - 127)[..., None]
        x, z = s["q"][row:row + ql].double(), s["lse"][row:row + ql].double()
        row += ql
        i = torch.arange(kv - ql, kv, device=DEV)[:, None]
        j = torch.arange(kv, device=DEV)[None, :]
        hidden = j > i
        if case["window"]:
            hidden |= (i - j >= case["window"]) & (j >= case["sinks"])
        at = torch.arange(kv, device=DEV)
        for c in range(n_kv):
            kc = k[:, c].reshape(-1, hd)[:kv]
            new = torch.where(at < kv - ql, out[ids[at // ps], c, at % ps], 0.0)
            for h in range(c * n_heads // n_kv, (c + 1) * n_heads // n_kv):
                p = torch.exp(x[:, h] @ kc.T * hd ** -0.5 - z[:, h:h + 1])
                new = new + p.masked_fill(hidden, 0.0).sum(0)
            out[ids[at // ps], c, at % ps] = new
    return out


def _exact_evict(s, kv_lens):
    case, ps, n_kv = s["case"], s["case"]["page"], _HEADS[s["case"]["heads"]][1]
    keep, sinks, recent = case["keep"], case["sinks"], case["recent"]
    names = [n for n in ("k_pages", "v_pages", "k_scales", "v_scales", "weights") if s[n] is not None]
    pools = {n: s[n].double().cpu() for n in names}
    old = {n: p.clone() for n, p in pools.items()}
    scores, table = s["scores"].cpu(), s["table"].long().cpu()
    for b, n in enumerate(kv_lens):
        if n <= keep:
            continue
        at = torch.arange(n)
        for h in range(n_kv):
            w = scores[table[b, at // ps], h, at % ps]
            order = torch.sort(-w[sinks:n - recent], stable=True).indices + sinks
            order = set(order[:keep - sinks - recent].tolist())
            late = iter(sorted(j for j in order if j >= keep - recent))
            to, of = [], []
            for j in range(sinks, keep - recent):
                if j not in order:
                    to.append(j)
                    of.append(next(late))
            to = torch.tensor(to + list(range(keep - recent, keep)), dtype=torch.long)
            of = torch.tensor(of + list(range(n - recent, n)), dtype=torch.long)
            for p in names:
                pools[p][table[b, to // ps], h, to % ps] = old[p][table[b, of // ps], h, of % ps]
    return {"kept": None, **{n: p if s[n].dtype != torch.uint8 else p.to(torch.uint8) for n, p in pools.items()}}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rotate":
        return tuple(_exact_turned(s, s[n], gain, s["positions"]) for n, gain in zip("qk", s["gains"]))
    if case["kind"] == "logprobs":
        return _exact_logprobs(s)
    q_lens, kv_lens = _lens(case)
    if case["kind"] == "append":
        return _exact_append(s, q_lens, kv_lens)
    return _exact_weigh(s, q_lens, kv_lens) if case["kind"] == "weigh" else _exact_evict(s, kv_lens)
