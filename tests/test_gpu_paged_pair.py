"""A model pair decoded over paged caches (paged_pair.py) against EAD, which keeps its own."""
import numpy as np
import pytest
import torch

import oracle
import paged_pair
import paper_2502_06833_amd as ead
import synth_inputs as si

pytestmark = pytest.mark.gpu

PROMPTS, NEW, D_MIN = (5, 40, 23), 40, 4


def _setup(dtype, **kw):
    Ws, Wl = (si.model_weights_torch(s, 0, "cuda") for s in (si.TINY_S, si.TINY_L))
    models = [paged_pair.PagedModel(s, w, dtype, **kw) for s, w in ((si.TINY_S, Ws), (si.TINY_L, Wl))]
    prompts = [si.prompt_np(0, f"pp{i}", n, si.TINY_S.vocab) for i, n in enumerate(PROMPTS)]
    return Ws, Wl, models, prompts


def test_the_same_tokens_as_the_handle():
    """Float32 pages: sequences admitted at different steps, prompts in pieces of 7, every token, model and entropy."""
    Ws, Wl, models, prompts = _setup(torch.float32)
    e = ead.EAD(si.TINY_S, Ws, si.TINY_L, Wl, window=5, tau=1e30, d_min=D_MIN, max_batch=3, max_seq=128)
    tau = float(np.median(e.generate(prompts, NEW)["Hbar"]))
    e.set_gate(5, tau, D_MIN)
    want = e.generate(prompts, NEW)
    e.close()
    assert 0.1 < want["model_id"].mean() < 0.9
    out, kept, _ = paged_pair.run(models, prompts, [0, 2, 9], NEW, tau=tau, d_min=D_MIN, piece=7, keep=torch.bfloat16)
    for i, o in enumerate(out):
        assert np.abs(np.array(o["H"]) - want["H"][i]).max() < 1e-3
        assert (np.array(o["tokens"]) == want["tokens"][i]).all() and (np.array(o["model_id"]) == want["model_id"][i]).all()
    assert sorted(kept) == [0, 1, 2] and all(len(m.free) == 256 and not m.pages for m in models)
    # what was handed over is the cache's own values, rounded
    k, v = kept[1][0][0].read(kept[1][0][1], torch.float32)
    assert k.shape[1:] == (4, 32) and bool(torch.isfinite(k).all()) and bool(torch.isfinite(v).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
def test_entropies_over_rounded_pages(dtype):
    """16- and 8-bit pages: the small model's first entropies stay near the float32 ones of the same text."""
    _, _, models, prompts = _setup(dtype)
    Ws = si.model_weights_torch(si.TINY_S, 0, "cuda")
    exact = paged_pair.PagedModel(si.TINY_S, Ws, torch.float32)
    feeds = [(i, list(map(int, p))) for i, p in enumerate(prompts)]
    h, _ = ead.entropy_argmax(models[0].feed(feeds))
    ref, _ = ead.entropy_argmax(exact.feed(feeds))
    # 8-bit keys and values are off by 2^-4 of themselves at most, and these models' logits spread by less than 1/4
    assert float((h - ref).abs().max()) < 2e-2


def test_pages_behind_a_window_are_given_back():
    _, _, models, prompts = _setup(torch.float32, n_pages=12, window=20, sinks=4)
    out, _, _ = paged_pair.run(models, prompts, [0, 2, 9], NEW, tau=-1e30, d_min=1000, piece=8)
    assert all(len(o["tokens"]) == NEW for o in out)
    # 80 positions of three sequences are 15 pages; a window of 20 and its sinks hold four a sequence
    assert len(models[0].free) == 12
