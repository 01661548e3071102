"""Beam search with a small random decoder, as the library's decoding operators are used together:

  paged attention of the newest tokens -> logits -> log probabilities and the best alternatives of every beam
  -> `profk.topk` over each search's beams x alternatives -> fork of the chosen beams' cache pages -> append -> ...

    python examples/beam_search.py [--searches 4] [--beams 4] [--steps 24] [--vocab 5003]

All state stays on the GPU; the loop reads nothing back until the end.  `dense_scores` computes the scores of finished
sequences again without a cache, in 64 bits."""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_12573_b200 as profk  # noqa: E402


class Decoder:
    """Attention layers with a residual around each, and nothing else: enough to need a cache."""

    def __init__(self, vocab: int, layers: int = 2, heads: int = 8, kv_heads: int = 2, dim: int = 64, seed: int = 0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        width = heads * dim

        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=g, device="cuda") * cols ** -0.5).to(torch.bfloat16)

        self.vocab, self.layers, self.heads, self.kv_heads, self.dim = vocab, layers, heads, kv_heads, dim
        self.embed, self.unembed = weight(vocab, width) * width ** 0.5, weight(vocab, width) * 4
        self.q = [weight(width, width) for _ in range(layers)]
        self.k = [weight(kv_heads * dim, width) for _ in range(layers)]
        self.v = [weight(kv_heads * dim, width) for _ in range(layers)]
        self.o = [weight(width, width) for _ in range(layers)]

    def step(self, tokens, pool, tables, lengths):
        """Logits of the tokens that follow `tokens` (one per sequence), whose keys and values go into the cache."""
        x = self.embed[tokens]
        for n in range(self.layers):
            q = (x @ self.q[n].t()).view(-1, self.heads, self.dim)
            k, v = ((x @ w[n].t()).view(-1, self.kv_heads, self.dim) for w in (self.k, self.v))
            profk.pages_append(pool[n, 0], pool[n, 1], tables, lengths, k, v)
            out, _ = profk.paged_attention(q, pool[n, 0], pool[n, 1], tables, lengths)
            x = x + out.flatten(1) @ self.o[n].t()
        return x @ self.unembed.t()

    def dense_scores(self, sequences):
        """Sum of the log probabilities of each sequence's tokens behind the first, without a cache and in 64 bits."""
        n, t = sequences.shape
        x = self.embed.double()[sequences]
        causal = torch.ones(t, t, dtype=torch.bool, device="cuda").tril()
        for i in range(self.layers):
            q, k, v = ((x @ w[i].double().t()).view(n, t, -1, self.dim).transpose(1, 2) for w in (self.q, self.k, self.v))
            k, v = (a.repeat_interleave(self.heads // self.kv_heads, 1) for a in (k, v))
            p = torch.softmax((q @ k.transpose(2, 3) * self.dim ** -0.5).masked_fill(~causal, float("-inf")), -1)
            x = x + (p @ v).transpose(1, 2).flatten(2) @ self.o[i].double().t()
        logp = torch.log_softmax(x @ self.unembed.double().t(), -1)
        return logp[:, :-1].gather(2, sequences[:, 1:, None]).sum((1, 2))


def beam_search(model: Decoder, first, beams: int, steps: int, page_size: int = 16, check: bool = False):
    """Searches from each token of `first`.  Returns (sequences (searches, beams, steps + 1), scores (searches, beams),
    refs, tables, lengths): the best `beams` continuations of each, best first, and the cache's state."""
    searches, dev = first.shape[0], first.device
    n, width = searches * beams, -(-(steps + 1) // page_size)
    pages = n * (width + 2)                                      # room for the old and the new last pages of every beam
    pool = torch.zeros(model.layers, 2, pages, model.kv_heads, page_size, model.dim, dtype=torch.bfloat16, device=dev)
    refs = torch.zeros(pages, dtype=torch.int32, device=dev)
    # one sequence per search to begin with: a fork of nothing
    state = profk.pages_fork(pool, torch.zeros(0, width, dtype=torch.int32, device=dev), refs[:0], refs,
                             torch.full((searches,), -1, dtype=torch.int32, device=dev), grow=1)
    missing = state.missing
    tokens, scores, alive = first, torch.zeros(searches, 1, device=dev), 1
    history = first[:, None]                                     # (searches * alive, tokens so far)
    base = torch.arange(searches, device=dev)[:, None]
    for _ in range(steps):
        logits = model.step(tokens, pool, state.tables, state.lengths)
        r = profk.logprobs(logits, k=beams, entropy=False)
        # each search's beams x alternatives, and the best of them
        total = (scores[:, :, None] + r.top_logprobs.view(searches, alive, beams)).view(searches, alive * beams)
        scores, pick = profk.topk(total, beams)
        parents = base * alive + pick // beams
        tokens = r.top_tokens.view(searches, -1).gather(1, pick).flatten()
        history = torch.cat([history[parents.flatten()], tokens[:, None]], 1)
        state = profk.pages_fork(pool, state.tables, state.lengths, state.refs, parents.flatten().to(torch.int32), grow=1)
        missing = missing + state.missing
        alive = beams
    if check:
        assert int(missing) == 0, "the pool ran out of pages"
    return history.view(searches, beams, -1), scores, state.refs, state.tables, state.lengths


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--searches", type=int, default=4)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--steps", type=int, default=24)
    ap.add_argument("--vocab", type=int, default=5003)
    a = ap.parse_args()
    model = Decoder(a.vocab)
    first = torch.arange(1, a.searches + 1, device="cuda")
    with torch.no_grad():
        sequences, scores, *_ = beam_search(model, first, a.beams, a.steps, check=True)
        again = model.dense_scores(sequences.flatten(0, 1)).view_as(scores)
    for s in range(a.searches):
        print(f"search {s}: best score {scores[s, 0]:.3f} (without a cache, in 64 bits: {again[s, 0]:.3f}), tokens {sequences[s, 0].tolist()}")


if __name__ == "__main__":
    main()
