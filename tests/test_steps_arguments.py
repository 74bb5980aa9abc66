"""What rotation, append, weighing, eviction and log probabilities refuse, without a GPU: the C entry points on descriptors, the Python ones on stand-ins."""
import ctypes as C

import pytest
import torch

import paper_2502_06833_amd as ead
from paper_2502_06833_amd import paged, rotary, scoring
from test_paged_arguments import OnGpu, batch_of, cache_of

OK, INVALID, SHAPE = 0, 1, 2
ROWS = paged.Rows(0x10000, 1024, 128)


def cache(**kw):
    f = dict(dtype=1, n_pages=8, page_size=16, n_kv_heads=2, head_dim=64, k=0x1000, v=0x2000, k_scale=None, v_scale=None)
    f.update(kw)
    return paged.CacheDesc(**f)


def batch(**kw):
    f = dict(batch=2, rows=4, max_q=2, min_q=1, max_kv=100, table_stride=8, table_width=8, page_table=0x3000, q_starts=0x4000, kv_lens=0x5000)
    f.update(kw)
    return paged.BatchDesc(**f)


def plan(**kw):
    f = dict(head_dim=64, rotary_dim=64, interleaved=0, gain_per_head=0, eps=1e-6, inv_freq=0x6000, q_gain=None, k_gain=None)
    f.update(kw)
    return rotary.RotaryDesc(**f)


def refused(rc, status, *words):
    assert rc == status, (rc, ead.lib().ead_last_error(None))
    if status:
        text = ead.lib().ead_last_error(None).decode()
        assert all(w in text for w in words), text


# Every call below is refused, or has nothing to do: none touches a GPU.
@pytest.mark.parametrize("bad,status,word", [
    (dict(head_dim=48), SHAPE, "head_dim"), (dict(head_dim=256), SHAPE, "head_dim"), (dict(rotary_dim=72), SHAPE, "rotary_dim"), (dict(rotary_dim=24), SHAPE, "rotary_dim"),
    (dict(rotary_dim=-16), SHAPE, "rotary_dim"), (dict(inv_freq=None), INVALID, "inv_freq"), (dict(inv_freq=0x6004), INVALID, "aligned"), (dict(q_gain=0x7002), INVALID, "aligned"),
    (dict(eps=-1.0), INVALID, "eps"), (dict(eps=float("nan")), INVALID, "eps"), (dict(eps=float("inf")), INVALID, "eps"),
])
def test_rotary_plans(bad, status, word):
    L, r = ead.lib(), plan(**bad)
    refused(L.ead_rotate(C.byref(r), 1, 4, 8, 2, 0x8000, C.byref(ROWS), C.byref(ROWS), C.byref(ROWS), C.byref(ROWS), None), status, word)
    c, b = cache(), batch()
    refused(L.ead_paged_append(C.byref(c), C.byref(b), C.byref(r), 1, 8, None, C.byref(ROWS), C.byref(ROWS), C.byref(ROWS), C.byref(ROWS), None), status, word)


def test_rotate_arguments():
    L, r, p = ead.lib(), plan(), C.byref
    call = lambda dtype=1, rows=4, h=8, kv=2, at=0x8000, q=ROWS, k=ROWS, qo=ROWS, ko=ROWS, r=r: L.ead_rotate(  # noqa: E731
        p(r) if r else None, dtype, rows, h, kv, at, p(q) if q else None, p(k) if k else None, p(qo) if qo else None, p(ko) if ko else None, None)
    refused(call(r=None), INVALID, "rotary")
    refused(call(dtype=2), INVALID, "dtype")
    refused(call(rows=-1), INVALID)
    refused(call(h=0, kv=0), INVALID)
    refused(call(h=-1), INVALID)
    refused(call(rows=1 << 28, h=8), SHAPE, "2^30")
    refused(call(at=None), INVALID, "positions")
    for name in ("q", "k", "qo", "ko"):
        refused(call(**{name: None}), INVALID)
        refused(call(**{name: paged.Rows(None, 64, 64)}), INVALID)
        refused(call(**{name: paged.Rows(0x10001, 64, 64)}), INVALID, "aligned")
    refused(call(rows=0, q=None, k=None, qo=None, ko=None, at=None), OK)


def test_append_arguments():
    L, r, p = ead.lib(), plan(), C.byref
    call = lambda c=None, b=None, r=r, dtype=1, h=8, q=ROWS, k=ROWS, v=ROWS, o=ROWS: L.ead_paged_append(  # noqa: E731
        p(c or cache()), p(b or batch()), p(r), dtype, h, None, p(q) if q else None, p(k) if k else None, p(v) if v else None, p(o) if o else None, None)
    refused(call(c=cache(head_dim=128)), SHAPE, "head_dim")
    refused(call(c=cache(dtype=2)), INVALID, "k_scale")
    refused(call(c=cache(page_size=24)), SHAPE, "page_size")
    refused(call(b=batch(max_q=5)), INVALID)
    refused(call(b=batch(kv_lens=None)), INVALID)
    refused(call(dtype=2), INVALID, "dtype")
    refused(call(h=-1), INVALID, "n_heads")
    for name in "qkvo":
        refused(call(**{name: None}), INVALID)
    refused(call(b=batch(rows=0, max_q=0, min_q=0), q=None, k=None, v=None, o=None), OK)


def test_weigh_arguments():
    L, p, n = ead.lib(), C.byref, C.c_uint64(0)
    at = lambda h=4, dtype=1, window=0, sinks=0, scale=0.1: paged.AttnDesc(h, dtype, window, sinks, scale, 0)  # noqa: E731
    size = lambda c=None, b=None, a=None: L.ead_paged_weigh_workspace(p(c or cache()), p(b or batch()), p(a or at()), p(n))  # noqa: E731
    assert size() == OK and n.value == 0
    assert size(b=batch(rows=6000, max_q=3000, max_kv=5000, table_stride=400, table_width=400)) == OK
    need = n.value
    assert need > 0 and need % 16 == 0
    for bad in (at(h=3), at(h=0), at(h=2 * 65)):
        refused(size(a=bad), SHAPE, "n_heads")
    for bad in (at(dtype=0), at(window=-1), at(sinks=-1), at(scale=0.0), at(scale=float("nan")), at(scale=3e38)):
        refused(size(a=bad), INVALID)
    refused(size(c=cache(dtype=0), a=at(dtype=1)), INVALID)
    call = lambda b=None, q=ROWS, lse=0x9000, w=0xA000, ws=None, size=0: L.ead_paged_weigh(p(cache()), p(b or batch()), p(at()), p(q) if q else None, lse, w, ws, size, None)  # noqa: E731
    refused(call(q=None), INVALID)
    refused(call(lse=None), INVALID, "lse")
    refused(call(w=None), INVALID, "weights")
    refused(call(w=0xA002), INVALID, "aligned")
    big = batch(rows=6000, max_q=3000, max_kv=5000, table_stride=400, table_width=400)
    refused(call(b=big), INVALID, "workspace")
    refused(call(b=big, ws=0xB000, size=need - 1), INVALID, str(need))
    refused(call(b=big, ws=0xB008, size=need), INVALID, "aligned")
    refused(call(b=batch(rows=0, max_q=0, min_q=0), q=None, lse=None, w=None), OK)


def test_evict_arguments():
    L, p, n = ead.lib(), C.byref, C.c_uint64(0)
    ev = lambda keep=32, sinks=2, recent=8: paged.EvictionDesc(keep, sinks, recent)  # noqa: E731
    size = lambda e, b=None: L.ead_paged_evict_workspace(p(cache()), p(b or batch()), p(e), p(n))  # noqa: E731
    assert size(ev()) == OK and n.value >= 4 * 4 + 4 * 22 * 8
    need = n.value
    for bad in (ev(keep=0), ev(keep=-5), ev(sinks=-1), ev(recent=-1), ev(sinks=30, recent=3), ev(sinks=2 ** 31 - 1, recent=2 ** 31 - 1)):
        refused(size(bad), INVALID, "eviction")
    refused(size(ev(), batch(max_kv=2 ** 20 + 1, table_width=2 ** 17, table_stride=2 ** 17)), SHAPE, "2^20")
    assert size(ev(), batch(max_kv=2 ** 20 + 1)) == OK                       # the table reaches 128 positions
    call = lambda s=0xA000, w=0xA000, k=0xB000, ws=0xC000, size=need: L.ead_paged_evict(p(cache()), p(batch()), p(ev()), s, w, k, ws, size, None)  # noqa: E731
    refused(call(s=None), INVALID, "scores")
    refused(call(s=0xA004), INVALID, "16-byte")
    refused(call(k=None), INVALID, "kept")
    refused(call(k=0xB001), INVALID, "aligned")
    refused(call(w=0xA002), INVALID, "aligned")
    refused(call(ws=None), INVALID, "workspace")
    refused(call(size=need - 1), INVALID, str(need))


def test_logprobs_arguments():
    L, p, n = ead.lib(), C.byref, C.c_uint64(0)

    def desc(**kw):
        f = dict(logits=0x10000, dtype=1, rows=4, vocab=1000, row_stride=1000, tokens=0x20000, top=5, unit=0, logprob=0x21000, H=0x22000, rank=0x23000, top_tokens=0x24000,
                 top_logprobs=0x25000)
        f.update(kw)
        return scoring.CallDesc(**f)

    for bad, status in ((dict(dtype=2), INVALID), (dict(rows=-1), SHAPE), (dict(rows=2 ** 22 + 1), SHAPE), (dict(vocab=0), SHAPE), (dict(vocab=2 ** 24 + 1), SHAPE), (dict(top=33), INVALID),
                        (dict(top=-1), INVALID), (dict(vocab=4, top=5), INVALID), (dict(unit=2), INVALID), (dict(row_stride=-1), INVALID)):
        d = desc(**bad)
        refused(L.ead_logprobs_workspace(p(d), p(n)), status)
        refused(L.ead_logprobs(p(d), None, 0, None), status)
    for bad in (dict(logits=None), dict(logits=0x10001), dict(tokens=None), dict(top_tokens=None), dict(top_logprobs=None), dict(tokens=0x20002), dict(H=0x22001), dict(rank=0x23003)):
        d = desc(**bad)
        refused(L.ead_logprobs(p(d), 0x30000, 1 << 30, None), INVALID)
    refused(L.ead_logprobs(None, None, 0, None), INVALID, "null")
    d = desc(vocab=151936, row_stride=151936)
    assert L.ead_logprobs_workspace(p(d), p(n)) == OK and n.value > 0
    refused(L.ead_logprobs(p(d), None, 0, None), INVALID, str(n.value))
    refused(L.ead_logprobs(p(d), 0x30000, n.value - 1, None), INVALID, "workspace")
    refused(L.ead_logprobs(p(d), 0x30008, n.value, None), INVALID, "aligned")
    refused(L.ead_logprobs(p(desc(rows=0, logits=None)), None, 0, None), OK)


# ---- the Python forms
@pytest.fixture
def host(monkeypatch):
    """Streams and devices without a GPU; a call that gets as far as the library fails the test."""
    for m in (paged, rotary, scoring):
        if hasattr(m, "_stream_ptr"):
            monkeypatch.setattr(m, "_stream_ptr", lambda: 0)
    monkeypatch.setattr(paged, "_current_device", lambda: 0)
    monkeypatch.setattr(rotary, "_current_device", lambda: 0)
    monkeypatch.setattr(paged, "_capturing", lambda: False)


class OnGpuToo(OnGpu):
    """... whose copies are there too."""

    def to(self, **kw):
        return OnGpuToo(self.t.to(dtype=kw["dtype"]), str(self.device))

    def contiguous(self):
        return self


def rot(**kw):
    freq = OnGpuToo(torch.ones(32, dtype=torch.float64))
    return ead.Rotary(64, inv_freq=freq, **kw)


def t(*shape, dtype=torch.bfloat16, device="cuda:0"):
    return OnGpu(torch.zeros(shape, dtype=dtype), device)


def test_rotary_refuses(host):
    for kw in (dict(head_dim=48), dict(head_dim=64, rotary_dim=65), dict(head_dim=64, rotary_dim=-16), dict(head_dim=64, theta=0.0)):
        with pytest.raises(ValueError):
            ead.Rotary(kw.pop("head_dim"), device="cpu", **kw)
    g = lambda *s, **kw: OnGpu(torch.ones(s, **kw))  # noqa: E731
    for q, k in ((g(32), None), (g(64, dtype=torch.float64), None), (g(64), g(2, 64)), (torch.ones(64), None), (OnGpu(torch.ones(64, 2).T[:1]), None),
                 (g(64), OnGpu(torch.ones(64), "cuda:1"))):
        with pytest.raises(ValueError):
            rot(q_gain=q, k_gain=k)
    with pytest.raises(ValueError):
        ead.Rotary(64, inv_freq=OnGpuToo(torch.ones(16)))
    r = rot()
    pos = t(3, dtype=torch.int32)
    for q, k, p in ((t(3, 4, 32), t(3, 2, 64), pos), (t(3, 4, 64), t(2, 2, 64), pos), (t(3, 4, 64), t(3, 2, 64, dtype=torch.float32), pos), (t(3, 256), t(3, 2, 64), pos),
                    (t(3, 4, 64), t(3, 2, 64), t(3, dtype=torch.int64)), (t(3, 4, 64), t(3, 2, 64), t(4, dtype=torch.int32)), (t(3, 4, 64), t(3, 2, 64), t(3, dtype=torch.int32, device="cuda:1")),
                    (t(3, 4, 64, device="cuda:1"), t(3, 2, 64), pos)):
        with pytest.raises(ValueError):
            r(q, k, p, out=(q, k))
    with pytest.raises((TypeError, ValueError)):
        r(t(3, 4, 64, dtype=torch.float16), t(3, 2, 64, dtype=torch.float16), pos)
    q, k = t(3, 4, 64), t(3, 2, 64)
    with pytest.raises(ValueError):
        r(q, k, pos, out=(OnGpu(torch.zeros(64, dtype=torch.bfloat16).expand(3, 4, 64)), k))
    with pytest.raises(ValueError):
        r(q, k, pos, out=(t(3, 4, 64, dtype=torch.float32), k))
    with pytest.raises(ValueError):
        rot(q_gain=g(5, 64), k_gain=g(2, 64))(q, k, pos, out=(q, k))


def test_steps_refuse_other_tensors(host):
    c, b, r = cache_of(), batch_of(torch.zeros(2, 3, dtype=torch.int32)), rot()
    q, kv, lse, w = t(2, 4, 64), t(2, 2, 64), t(2, 4, dtype=torch.float32), t(4, 2, 16, dtype=torch.float32)
    for args in ((t(2, 256), kv, kv), (q, t(2, 3, 64), kv), (q, kv, t(3, 2, 64)), (q, t(2, 2, 64, dtype=torch.float32), kv), (q, kv, t(2, 2, 64, device="cuda:1"))):
        with pytest.raises(ValueError):
            c.append(*args, b, r, out=q)
    for kw in (dict(out=t(2, 4, 64, dtype=torch.float32)), dict(out=OnGpu(torch.zeros(64, dtype=torch.bfloat16).expand(2, 4, 64))), dict(out=q, positions=t(2, dtype=torch.int64)),
               dict(out=q, positions=t(3, dtype=torch.int32))):
        with pytest.raises(ValueError):
            c.append(q, kv, kv, b, r, **kw)
    for args in ((t(2, 4, 64, dtype=torch.float32), lse, b, w), (q, t(2, 4), b, w), (q, t(2, 5, dtype=torch.float32), b, w), (q, OnGpu(torch.zeros(4, 2).T), b, w),
                 (q, lse, b, t(4, 2, 16)), (q, lse, b, t(4, 2, 8, dtype=torch.float32)), (q, lse, b, t(4, 2, 16, dtype=torch.float32, device="cuda:1")),
                 (q, lse, batch_of(torch.zeros(2, 3, dtype=torch.int32), "cuda:1"), w), (q, lse, b, OnGpu(torch.zeros(4, 2, 32)[:, :, ::2]))):
        with pytest.raises(ValueError):
            c.weigh(*args)
    for bad in (2 ** 31, -2 ** 31 - 1):
        with pytest.raises(ValueError):
            c.weigh(q, lse, b, w, window=bad)
        with pytest.raises(ValueError):
            c.evict(b, w, bad)
    for kw in (dict(keep=0), dict(keep=4, sinks=3, recent=2), dict(keep=4, sinks=-1), dict(keep=4, recent=-1), dict(keep=4, weights=t(4, 2, 8, dtype=torch.float32)),
               dict(keep=4, kept=t(2, 2, 4)), dict(keep=4, kept=t(2, 2, 5, dtype=torch.int32)), dict(keep=4, kept=OnGpu(torch.zeros(2, 4, 2, dtype=torch.int32).transpose(1, 2)))):
        with pytest.raises(ValueError):
            c.evict(b, w, **kw)
    with pytest.raises(ValueError):
        c.evict(b, t(4, 2, 16), 4)


def test_logprobs_refuses(host):
    x, tok = t(3, 100), t(3, dtype=torch.int32)
    for args, kw in (((torch.zeros(3, 100),), {}), ((t(300),), {}), ((OnGpu(torch.zeros(100, 3).T),), {}), ((x, t(3, dtype=torch.int64)), {}), ((x, t(4, dtype=torch.int32)), {}),
                     ((x, t(3, dtype=torch.int32, device="cuda:1")), {}), ((x, tok), dict(top=33)), ((x, tok), dict(top=-1)), ((t(3, 4), tok), dict(top=5)), ((t(3, 0),), {}),
                     ((t(3, 100, device="cuda:1"),), {})):
        with pytest.raises(ValueError):
            ead.logprobs(*args, **kw)
    with pytest.raises(TypeError):
        ead.logprobs(t(3, 100, dtype=torch.float16))
