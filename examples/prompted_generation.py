"""Answers to ragged prompts with a small random decoder, as the library's operators for prompts and drafts are used together:

  prompts in parts: `profk.pages_append_rotary` -> `profk.paged_attention_chunk` -> ... -> logits of each prompt's last token
  every token: `profk.adjust_logits` (repetition, presence, a grammar's mask) -> `profk.logprobs` -> the best token ->
               `profk.pages_append_rotary` -> `profk.paged_attention` -> logits -> ...
  drafts:      several tokens of every sequence at a time through the same cache, all their logits at once
  training:    the same model without a cache, `profk.rotary` and `profk.logprobs` with their gradients

    python examples/prompted_generation.py [--prompts 4] [--steps 16] [--part 64] [--vocab 5003]

All state stays on the GPU; the loops read nothing back until the end."""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_12573_b200 as profk  # noqa: E402


class Decoder:
    """Attention layers with rotary positions (of half of each head) and a residual around each."""

    def __init__(self, vocab: int, layers: int = 2, heads: int = 8, kv_heads: int = 2, dim: int = 64, interleaved: bool = False, seed: int = 0,
                 dtype=torch.bfloat16):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        width = heads * dim

        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=g, device="cuda") * cols ** -0.5).to(dtype)

        self.vocab, self.layers, self.heads, self.kv_heads, self.dim, self.interleaved = vocab, layers, heads, kv_heads, dim, interleaved
        self.embed, self.unembed = weight(vocab, width) * width ** 0.5, weight(vocab, width) * 4
        # queries, keys and values from one product
        self.qkv = [weight((heads + 2 * kv_heads) * dim, width) for _ in range(layers)]
        self.o = [weight(width, width) for _ in range(layers)]
        self.frequencies = profk.rotary_frequencies(dim // 2)

    def heads_of(self, x, n):
        joint = (x @ self.qkv[n].t()).unflatten(-1, (-1, self.dim))
        return joint.split([self.heads, self.kv_heads, self.kv_heads], -2)

    def hidden(self, tokens, pool, tables, lengths, starts=None):
        """The last layer's output for new `tokens` of every sequence: (seqs,), (seqs, n), or with `starts` (rows,).  Their keys and
        values go into the cache; `lengths` counts them already."""
        x = self.embed[tokens]
        for n in range(self.layers):
            q, k, v = self.heads_of(x, n)
            q = profk.pages_append_rotary(pool[n, 0], pool[n, 1], tables, lengths, q, k, v, self.frequencies, starts=starts, interleaved=self.interleaved)
            if starts is None and tokens.dim() == 1:
                out, _ = profk.paged_attention(q, pool[n, 0], pool[n, 1], tables, lengths)
            else:
                out, _ = profk.paged_attention_chunk(q, pool[n, 0], pool[n, 1], tables, lengths, starts=starts)
            x = x + out.flatten(-2) @ self.o[n].t()
        return x

    def logits(self, x):
        return x @ self.unembed.t()

    def dense_logits(self, sequences):
        """The same of whole `sequences` (n, t) without a cache, differentiable in the weights."""
        t = sequences.shape[1]
        x = self.embed[sequences]
        places, late = torch.arange(t, device="cuda"), torch.ones(t, t, dtype=torch.bool, device="cuda").triu(1)
        for n in range(self.layers):
            q, k, v = self.heads_of(x, n)
            q, k = (profk.rotary(a, places, self.frequencies, interleaved=self.interleaved) for a in (q, k))
            q, k, v = (a.transpose(1, 2) for a in (q, k, v))
            k, v = (a.repeat_interleave(self.heads // self.kv_heads, 1) for a in (k, v))
            p = torch.softmax((q @ k.transpose(2, 3) * self.dim ** -0.5).masked_fill(late, float("-inf")), -1)
            x = x + (p @ v).transpose(1, 2).flatten(2) @ self.o[n].t()
        return self.logits(x)

    def loss(self, sequences):
        """Mean negative log probability of every token behind the first."""
        r = profk.logprobs(self.dense_logits(sequences[:, :-1]), sequences[:, 1:].contiguous(), entropy=False)
        return -r.logprob.mean()


class Cache:
    """Pages for `room` tokens of each of `seqs` sequences."""

    def __init__(self, model: Decoder, seqs: int, room: int, page_size: int = 16):
        pages = seqs * -(-room // page_size)
        self.pool = torch.zeros(model.layers, 2, pages, model.kv_heads, page_size, model.dim, dtype=model.embed.dtype, device="cuda")
        nothing = torch.zeros(pages, dtype=torch.int32, device="cuda")
        state = profk.pages_fork(self.pool, torch.zeros(0, -(-room // page_size), dtype=torch.int32, device="cuda"), nothing[:0], nothing,
                                 torch.full((seqs,), -1, dtype=torch.int32, device="cuda"), grow=room)
        self.tables, self.refs, self.missing = state.tables, state.refs, state.missing
        self.lengths = torch.zeros_like(state.lengths)


def read_prompts(model: Decoder, prompts, cache: Cache, part: int):
    """Takes the prompts (lists of tokens) into the cache, at most `part` tokens of each at a time; the logits behind them."""
    last = [None] * len(prompts)
    for begin in range(0, max(len(p) for p in prompts), part):
        pieces = [p[begin:begin + part] for p in prompts]
        new = torch.tensor([len(p) for p in pieces], dtype=torch.int32, device="cuda")
        starts = torch.cat([new.new_zeros(1), torch.cumsum(new, 0, dtype=torch.int32)])
        cache.lengths = cache.lengths + new
        x = model.hidden(torch.tensor([t for p in pieces for t in p], device="cuda"), cache.pool, cache.tables, cache.lengths, starts)
        row = -1
        for i, p in enumerate(pieces):
            row += len(p)
            if p and begin + part >= len(prompts[i]):
                last[i] = x[row]
    return model.logits(torch.stack(last))


def generate(model: Decoder, prompts, steps: int, part: int = 64, page_size: int = 16, repetition: float = 1.2, presence: float = 0.3, mask=None):
    """`steps` tokens behind every prompt, the best one each time.  `mask`: a grammar's allowed tokens, as `adjust_logits` takes
    them.  Returns (tokens (seqs, longest + steps), lengths, cache, logits of each step (steps, seqs, vocab) as the selection saw them)."""
    seqs, longest = len(prompts), max(len(p) for p in prompts)
    cache = Cache(model, seqs, longest + steps, page_size)
    held = torch.tensor([len(p) for p in prompts], dtype=torch.int32, device="cuda")
    tokens = torch.zeros(seqs, longest + steps, dtype=torch.int64, device="cuda")
    for i, p in enumerate(prompts):
        tokens[i, :len(p)] = torch.tensor(p, device="cuda")
    logits, lengths, seen = read_prompts(model, prompts, cache, part), held.clone(), []
    for step in range(steps):
        profk.adjust_logits(logits, tokens, lengths, held, repetition=repetition, presence=presence, mask=mask, out=logits)
        seen.append(logits)
        best = profk.logprobs(logits, k=1, entropy=False).top_tokens[:, 0]
        tokens.scatter_(1, lengths.long()[:, None], best[:, None])
        lengths = lengths + 1
        if step + 1 < steps:
            cache.lengths = cache.lengths + 1
            logits = model.logits(model.hidden(best, cache.pool, cache.tables, cache.lengths))
    return tokens, lengths, cache, torch.stack(seen)


def check_drafts(model: Decoder, cache: Cache, drafts):
    """Logits behind every one of `drafts` (seqs, n), whose keys and values go behind what the cache holds.  (What is not kept of
    them is overwritten by the next tokens: its length is what the cache's holder says it is.)"""
    x = model.hidden(drafts, cache.pool, cache.tables, cache.lengths + drafts.shape[1])
    return model.logits(x)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--prompts", type=int, default=4)
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--part", type=int, default=64)
    ap.add_argument("--vocab", type=int, default=5003)
    a = ap.parse_args()
    g = torch.Generator()
    g.manual_seed(0)
    prompts = [torch.randint(0, a.vocab, (5 + 40 * i,), generator=g).tolist() for i in range(a.prompts)]
    model = Decoder(a.vocab)
    with torch.no_grad():
        tokens, lengths, cache, _ = generate(model, prompts, a.steps, a.part)
        assert int(cache.missing) == 0, "the pool ran out of pages"
    for i, p in enumerate(prompts):
        print(f"prompt of {len(p)} tokens: {tokens[i, len(p):int(lengths[i])].tolist()}")


if __name__ == "__main__":
    main()
