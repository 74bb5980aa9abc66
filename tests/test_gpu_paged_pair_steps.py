"""paged_pair.py within a budget of positions, and with alternatives to its tokens."""
import numpy as np
import pytest
import torch

import paged_pair
import paper_2502_06833_amd as ead
import synth_inputs as si

pytestmark = pytest.mark.gpu

PROMPTS, NEW = (5, 40, 23), 40


def models_of(dtype, **kw):
    models = [paged_pair.PagedModel(s, si.model_weights_torch(s, 0, "cuda"), dtype, **kw) for s in (si.TINY_S, si.TINY_L)]
    return models, [si.prompt_np(0, f"pp{i}", n, si.TINY_S.vocab) for i, n in enumerate(PROMPTS)]


def decode(models, prompts, **kw):
    return paged_pair.run(models, prompts, [0, 2, 9], NEW, tau=-1e30, d_min=6, piece=8, **kw)[0]


def test_alternatives_are_the_tokens_own():
    """The same tokens and entropies with them as without; the token comes first, its log probability is that of the text scored at once."""
    models, prompts = models_of(torch.float32)
    plain = decode(models, prompts)
    with_them = decode(models, prompts, top=4)
    for o, p in zip(with_them, plain):
        assert o["tokens"] == p["tokens"] and o["model_id"] == p["model_id"] and np.abs(np.array(o["H"]) - np.array(p["H"])).max() < 1e-5
        assert not p["alternatives"] and [t[0] for t, _ in o["alternatives"]] == o["tokens"]
        assert all(len(set(t)) == 4 and sorted(lp, reverse=True) == lp and lp[0] <= 0 for t, lp in o["alternatives"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float8_e4m3fn])
def test_a_budget_holds(dtype):
    """Pools that are too small for the whole texts: 80 positions of three sequences are 15 pages, a budget of 32 and a page more are nine."""
    models, prompts = models_of(dtype, n_pages=10, budget=32, sinks=2, recent=8)
    out = decode(models, prompts, top=1)
    assert all(len(o["tokens"]) == NEW for o in out) and all(np.isfinite(o["H"]).all() for o in out)
    assert all(len(m.free) == 10 and not m.pages and not m.gone for m in models)


def test_a_budget_that_is_never_reached_changes_nothing():
    models, prompts = models_of(torch.float32)
    whole = decode(models, prompts)
    models, prompts = models_of(torch.float32, budget=200, recent=8)
    assert [o["tokens"] for o in decode(models, prompts)] == [o["tokens"] for o in whole]


def test_what_is_kept_is_what_was_paid_most():
    """A cache cut once: attention over what is left is attention over those positions of the whole cache."""
    models, prompts = models_of(torch.float32, budget=24, sinks=2, recent=4)
    m, text = models[0], list(map(int, prompts[1]))
    m.feed([(0, text[:39])])
    assert m.have[0] == 39 and m.seen(0) == 39
    m.feed([(0, text[39:40])])
    assert m.have[0] == 24 and m.seen(0) == 40 and len(m.pages[0]) == 2
    whole = paged_pair.PagedModel(si.TINY_S, m.w, torch.float32)
    whole.feed([(0, text)])
    batch = [ead.PagedBatch.of([x.pages[0]], [x.have[0]], [x.have[0]]) for x in (m, whole)]
    for mine, theirs in zip(m.caches, whole.caches):
        a, b = mine.read(batch[0], torch.float32)[0], theirs.read(batch[1], torch.float32)[0]
        for h in range(a.shape[1]):
            # every vector that is left is one of the whole cache's, no two the same, the first two and the last four in their places
            d = (a[:, h, None] - b[None, :, h]).abs().amax(-1)
            of = d.argmin(1)
            assert float(d.amin(1).max()) < 1e-4 and of.unique().numel() == 24 and of[:2].tolist() == [0, 1] and of[-4:].tolist() == [36, 37, 38, 39]
