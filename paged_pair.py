#!/usr/bin/env python3
"""Entropy Adaptive Decoding over paged caches, with sequences that come and go (needs a GPU).

`EAD` owns its caches and takes a batch of prompts at a time.  A server with a scheduler of its own keeps them itself:
here both models of a pair hold their keys and values in pages (`PagedCache`, one per layer), sequences are admitted at
any step, their prompts are taken in pieces beside the other sequences' decode rows, and a model that takes over
catches up with the tokens the other one produced, all in one call of `write` and one of `attention` per layer.
Entropies and tokens come from `entropy_argmax`; the window mean and the switch rule (Eq. 3-4) are a few lines here.  A
finished sequence's cache is read back and written to a second cache in 8 bits, as one would hand it to another
program or keep it for a later turn.  With `--window` only the last positions and the first `--sinks` are attended to,
and pages that a window has left behind go back to the pool.

  python paged_pair.py [--cache f32|bf16|fp8] [--window 48 --sinks 4] [--sequences 6] [--new 48] [--piece 16]
"""
import argparse
import json
import sys
from collections import deque

import synth_inputs as si


class PagedModel:
    """One decoder of the pair: weights as in synth_inputs, a page table per sequence, a PagedCache per layer."""

    def __init__(self, shape, weights, cache_dtype, n_pages=256, page=16, window=0, sinks=0):
        import torch
        import paper_2502_06833_amd as ead
        self.s, self.w, self.page, self.window, self.sinks = shape, weights, page, window, sinks
        self.io = torch.float32 if cache_dtype == torch.float32 else torch.bfloat16
        self.caches = [ead.PagedCache.empty(n_pages, page, shape.n_kv_heads, shape.head_dim, cache_dtype) for _ in range(shape.n_layers)]
        self.free = list(range(n_pages))
        self.pages, self.have = {}, {}
        half = shape.head_dim // 2
        self.freq = float(shape.rope_theta) ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)

    def _grow(self, seq, n):
        """Room for n more positions; pages that no later row sees are given back."""
        pages = self.pages.setdefault(seq, [])
        have = self.have.get(seq, 0)
        while len(pages) * self.page < have + n:
            if not self.free:
                raise RuntimeError("no free page")
            pages.append(self.free.pop())
        if self.window:
            for i in range(-(-self.sinks // self.page), max(0, have - self.window + 1) // self.page):
                if pages[i] >= 0:
                    self.free.append(pages[i])
                    pages[i] = -1
        self.have[seq] = have + n

    def drop(self, seq):
        self.free += [p for p in self.pages.pop(seq, []) if p >= 0]
        self.have.pop(seq, None)

    def _norm(self, x, gain):
        return x * (x.square().mean(-1, keepdim=True) + self.s.rms_eps).rsqrt() * gain

    def _rotate(self, x, cos, sin):
        import torch
        a, b = x.chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    def feed(self, feeds):
        """feeds: (sequence, tokens it has not seen yet).  Float32 logits of every feed's last token."""
        import torch
        import paper_2502_06833_amd as ead
        s, w = self.s, self.w
        first = [self.have.get(q, 0) for q, _ in feeds]
        for q, t in feeds:
            self._grow(q, len(t))
        lens = [len(t) for _, t in feeds]
        batch = ead.PagedBatch.of([self.pages[q] for q, _ in feeds], lens, [self.have[q] for q, _ in feeds])
        ids = torch.tensor([x for _, t in feeds for x in t], device="cuda")
        pos = torch.tensor([p for f, n in zip(first, lens) for p in range(f, f + n)], device="cuda", dtype=torch.float64)
        angle = pos[:, None, None] * self.freq
        cos, sin = angle.cos().float(), angle.sin().float()
        mat = lambda a, name: a @ w[name].float().T  # noqa: E731
        x = w["embed"][ids].float()
        for l in range(s.n_layers):
            p = f"layers.{l}."
            a = self._norm(x, w[p + "norm_attn"])
            q = self._rotate(mat(a, p + "wq").view(-1, s.n_heads, s.head_dim), cos, sin)
            k = self._rotate(mat(a, p + "wk").view(-1, s.n_kv_heads, s.head_dim), cos, sin)
            v = mat(a, p + "wv").view(-1, s.n_kv_heads, s.head_dim)
            self.caches[l].write(k, v, batch)
            o = self.caches[l].attention(q.to(self.io), batch, window=self.window, sinks=self.sinks)
            x = x + mat(o.float().flatten(1), p + "wo")
            b = self._norm(x, w[p + "norm_ffn"])
            x = x + mat(torch.nn.functional.silu(mat(b, p + "w_gate")) * mat(b, p + "w_up"), p + "w_down")
        last = torch.tensor(lens, device="cuda").cumsum(0) - 1
        return mat(self._norm(x[last], w["norm_final"]), "lm_head").contiguous()

    def hand_over(self, seq, dtype):
        """The sequence's keys and values of every layer in a cache of its own and of another type."""
        import paper_2502_06833_amd as ead
        n = self.have[seq]
        mine = ead.PagedBatch.of([self.pages[seq]], [n], [n])
        count = -(-n // self.page)
        out, theirs = [], ead.PagedBatch.of([list(range(count))], [n], [n])
        for c in self.caches:
            k, v = c.read(mine, self.io)
            other = ead.PagedCache.empty(count, self.page, self.s.n_kv_heads, self.s.head_dim, dtype)
            other.write(k, v, theirs)
            out.append((other, theirs))
        return out


class Sequence:
    """Algorithm 1's state of one sequence."""

    def __init__(self, prompt, w, tau, d_min):
        self.text, self.prompt_len = list(map(int, prompt)), len(prompt)
        self.recent, self.tau, self.d_min = deque(maxlen=w), tau, d_min
        self.model, self.c = 0, 0
        self.out = {"tokens": [], "model_id": [], "H": [], "Hbar": []}

    def take(self, h, token):
        self.recent.append(h)
        mean = sum(self.recent) / len(self.recent)
        for name, x in (("tokens", token), ("model_id", self.model), ("H", h), ("Hbar", mean)):
            self.out[name].append(x)
        self.text.append(token)
        self.c += 1
        wanted = 1 if mean > self.tau else 0
        if self.c >= self.d_min and wanted != self.model:
            self.model, self.c = wanted, 0


def run(models, prompts, arrivals, new, w=5, tau=0.0, d_min=4, piece=16, keep=None):
    """Decode `new` tokens for every prompt, admitted at step arrivals[i]; prompts go in pieces of `piece` tokens.
    keep: a cache type finished sequences are handed over in.  Returns (outputs per prompt, caches handed over, steps)."""
    import paper_2502_06833_amd as ead
    seqs = [Sequence(p, w, tau, d_min) for p in prompts]
    kept, step, done = {}, 0, set()
    while len(done) < len(seqs):
        live = [i for i in range(len(seqs)) if arrivals[i] <= step and i not in done]
        for m in (0, 1):
            feeds = []
            for i in live:
                if seqs[i].model == m and len(seqs[i].out["tokens"]) < new:
                    seen = models[m].have.get(i, 0)
                    feeds.append((i, seqs[i].text[seen:seen + piece]))
            if not feeds:
                continue
            h, token = ead.entropy_argmax(models[m].feed(feeds))
            stays = {i for i, _ in feeds if models[m].have[i] < len(seqs[i].text)}       # more of its text to come
            for (i, _), hi, ti in zip(feeds, h.tolist(), token.tolist()):
                if i not in stays:
                    seqs[i].take(hi, ti)
            live = [i for i in live if i not in {j for j, _ in feeds}]                   # one step for each sequence
        for i, s in enumerate(seqs):
            if i not in done and len(s.out["tokens"]) >= new:
                done.add(i)
                if keep is not None and all(p >= 0 for p in models[0].pages[i]):         # nothing of it was given back
                    kept[i] = models[0].hand_over(i, keep)
                for model in models:
                    model.drop(i)
        step += 1
    return [s.out for s in seqs], kept, step


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--cache", choices=["f32", "bf16", "fp8"], default="fp8")
    ap.add_argument("--window", type=int, default=0)
    ap.add_argument("--sinks", type=int, default=0)
    ap.add_argument("--sequences", type=int, default=6)
    ap.add_argument("--new", type=int, default=48)
    ap.add_argument("--piece", type=int, default=16)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    import torch
    if not torch.cuda.is_available():
        sys.exit("paged_pair.py needs a GPU")
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}[a.cache]
    shapes = (si.TINY_S, si.TINY_L)
    models = [PagedModel(s, si.model_weights_torch(s, a.seed, "cuda"), dtype, window=a.window, sinks=a.sinks) for s in shapes]
    prompts = [si.prompt_np(a.seed, f"paged{i}", 7 + 11 * i, shapes[0].vocab) for i in range(a.sequences)]
    small, _, _ = run(models, prompts, [0] * a.sequences, a.new, tau=1e30, piece=a.piece)
    tau = sorted(x for o in small for x in o["Hbar"])[a.sequences * a.new // 2]
    out, kept, steps = run(models, prompts, [3 * i for i in range(a.sequences)], a.new, tau=tau, piece=a.piece, keep=torch.float8_e4m3fn)
    ids = [m for o in out for m in o["model_id"]]
    print(json.dumps({"cache": a.cache, "window": a.window, "sinks": a.sinks, "sequences": a.sequences, "new_tokens": len(ids), "steps": steps,
                      "tau": round(tau, 4), "large_share": round(sum(ids) / len(ids), 4), "handed_over": len(kept),
                      "free_pages": [len(m.free) for m in models]}))


if __name__ == "__main__":
    main()
