"""The forms that log probabilities of many rows and wide vocabularies take: several sets to a group whose largest logits are noted, long rows in float32, bounds of 0 and below.
Tolerances are those of test_gpu_logprobs."""
import math

import pytest
import torch

import paper_2502_06833_amd as ead
from test_gpu_logprobs import DEV, check, rows

pytestmark = pytest.mark.gpu


def check_rows(x, r, t, top, each=64):
    for i in range(0, x.shape[0], each):
        part = slice(i, i + each)
        check(x[part], type(r)(*(f[part] if f is not None else None for f in r)), t[part], top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,vocab,top", [(1030, 170001, 20), (1100, 333337, 32), (1025, 163841, 1)])        # whole rows to a workgroup: 21 sets to a wave and more
@pytest.mark.parametrize("shift", [0.0, -60.0])                                                            # (all logits below 0: so is the bound)
def test_many_rows_of_wide_vocabularies(dtype, n, vocab, top, shift):
    x, t = rows(n, vocab, dtype, seed=vocab)
    x += shift
    some = torch.randperm(n, device=DEV)[:128]
    r = ead.logprobs(x, t, top=top)
    check_rows(x[some], type(r)(*(f[some] for f in r)), t[some], top)
    # every row by its own sums: the same call of one row at a time is another form
    for i in range(0, n, 101):
        one = ead.logprobs(x[i:i + 1], t[i:i + 1], top=top)
        assert torch.equal(one.top_tokens[0], r.top_tokens[i]) and int(one.rank) == int(r.rank[i]) and abs(float(one.H - r.H[i])) < 1e-4


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 3, 40, 300, 520, 1030])
@pytest.mark.parametrize("top", [5, 32])
@pytest.mark.parametrize("shift", [0.0, -30.0])
def test_long_rows_of_every_cut(dtype, n, top, shift):
    """From a set or two to a wave (still in registers when the bound is known) to whole rows."""
    x, t = rows(n, 100003, dtype, seed=n)
    x += shift
    r = ead.logprobs(x, t, top=top)
    some = slice(0, 128)
    check_rows(x[some], type(r)(*(f[some] for f in r)), t[some], top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,vocab", [(1030, 170001), (8, 170001), (513, 60007)])
def test_kinds_of_rows(dtype, n, vocab):
    """Few distinct logits, masks, peaks that lie together, zeros of both signs, rows that fall and rise, in batches whose other rows are ordinary."""
    x, t = rows(n, vocab, dtype, seed=1)
    at = torch.arange(vocab, device=DEV)
    low = torch.finfo(dtype).min
    x[0] = 0.0
    x[1] = torch.where(at % 2 == 0, 0.0, -0.0).to(dtype)
    x[2] = -(at % 7).to(dtype)
    x[3] = torch.where((at > vocab - 200) & (at % 3 == 0), -1.0, -math.inf).to(dtype)          # 66 equal ones at the end, nothing else
    x[4] = torch.where(at == vocab - 1, -5.0, low).to(dtype)
    x[5] = (-at.float() / 1000).to(dtype)
    x[6] = (at.float() / 1000 - 1000).to(dtype)
    x[7, 5000:5040] = 30.0 - torch.arange(40, device=DEV).to(dtype) / 4                        # forty peaks in one wave's set
    t[:8] = torch.tensor([3, 4, 9, vocab - 2, vocab - 1, 70, 11, 5001], dtype=torch.int32, device=DEV)
    for top in (1, 7, 32):
        r = ead.logprobs(x, t, top=top)
        check_rows(x[:40], type(r)(*(f[:40] for f in r)), t[:40], top)


def test_a_million_logits_and_more():
    for n, vocab in ((1, 1 << 24), (2, 3_000_017), (70, 1_000_003)):
        for dtype in (torch.bfloat16, torch.float32):
            x, t = rows(n, vocab, dtype, seed=n)
            r = ead.logprobs(x, t, top=32)
            check_rows(x[:4], type(r)(*(f[:4] for f in r)), t[:4], 32, each=1)


def test_threads_on_one_stream():
    """Calls of four threads, every one of another size, on the stream that they share."""
    import threading
    data = [rows(n, 40009, torch.float32, seed=n) for n in (2, 30, 150, 700)]
    want = [ead.logprobs(x, t, top=9) for x, t in data]
    torch.cuda.synchronize()
    got, gate = [[] for _ in data], threading.Barrier(len(data))

    def work(i):
        gate.wait()
        for _ in range(25):
            got[i].append(ead.logprobs(*data[i], top=9))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(data))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert len(g) == 25 and all(torch.equal(a, b) for r in g for a, b in zip(w, r))
