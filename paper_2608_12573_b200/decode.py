"""The operators around a selection in a decoding loop: log probabilities with entropy and top alternatives (and their
gradient), the forking and compaction of the pages of a key-value cache, and attention of one token over them; and those that
take prompts and drafts into it: rotary positions (and their gradient), appending with them, attention of a chunk of new
tokens, and what is laid over logits before a selection.

Checks, allocation and marshalling are done by the in-tree extension module `_decode` (csrc/decode_binding.cpp), which calls
the C ABI of `profk.h`; a refusal raises `ProfkError`.  Of all of them `logprobs` and `rotary` have derivatives; the others refuse tensors
that require a gradient unless grad mode is off.  Nothing is synchronised, and scratch memory comes from torch's
allocator on the current stream, so that calls on several streams do not meet.
"""
from __future__ import annotations

import math
from typing import NamedTuple, Optional

import torch

_native = None


def _load():
    """The extension module; raises if it has not been built."""
    global _native
    if _native is None:
        import paper_2608_12573_b200 as package

        package.lib()
        try:
            from . import _decode
        except ImportError as e:
            raise package.ProfkError(f"the extension module _decode cannot be loaded ({e}): run "
                                     "paper_2608_12573_b200._build.build() (there is no fallback implementation)") from e
        _decode.set_errors(package.ProfkError, torch.OutOfMemoryError)
        _native = _decode
    return _native


class LogProbs(NamedTuple):
    """What `logprobs` returns; all but the tokens are float32.  A part that was not asked for is None."""
    logprob: Optional[torch.Tensor]         # (...)    of the given tokens
    lse: torch.Tensor                       # (...)    ln sum e^(logit / temperature)
    entropy: Optional[torch.Tensor]         # (...)
    top_logprobs: Optional[torch.Tensor]    # (..., k)
    top_tokens: Optional[torch.Tensor]      # (..., k) int64
    lse_rest: torch.Tensor                  # (...)    what the rounding of lse left off, for `logprobs_backward`


class _LogProbsGradient(torch.autograd.Function):
    """The gradient as a node of its own, for `create_graph=True`: a second derivative is refused, not left out."""
    @staticmethod
    def forward(ctx, *args):
        return _load().logprobs_backward(*args)

    @staticmethod
    def backward(ctx, *_):
        import paper_2608_12573_b200 as package

        raise package.ProfkError("logprobs can be differentiated once only")


class _LogProbsFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, k, temperature, entropy):
        r = LogProbs._make(_load().logprobs(logits, tokens, k, temperature, entropy))
        ctx.save_for_backward(logits, tokens, r.lse, r.lse_rest, r.entropy, r.top_tokens)
        ctx.temperature = temperature
        ctx.set_materialize_grads(False)
        ctx.mark_non_differentiable(*(t for t in (r.top_tokens, r.lse_rest) if t is not None))
        return tuple(r)

    @staticmethod
    def backward(ctx, g_logprob, g_lse, g_entropy, g_top, _tokens, _rest):
        logits, tokens, lse, rest, entropy, top = ctx.saved_tensors

        def dense(g):
            return None if g is None else g.contiguous()

        args = (logits, lse, rest, tokens, dense(g_logprob), entropy, dense(g_entropy), dense(g_lse), top, dense(g_top), ctx.temperature)
        # (grad mode is on here where a graph of the gradient was asked for)
        grad = _LogProbsGradient.apply(*args) if torch.is_grad_enabled() else _load().logprobs_backward(*args)
        return grad, None, None, None, None


def logprobs(logits, tokens=None, k: int = 0, temperature: float = 1.0, entropy: bool = True) -> LogProbs:
    """`profk_logprobs_*` on the current stream: log probabilities of `tokens`, log-sum-exp, entropy and the `k` most
    probable tokens of every row of `logits / temperature`, in one read of the logits.

    logits: CUDA tensor (..., V), float32, bfloat16 or float16, dense rows at any stride.  tokens: int64 (...), negative
    where no token is given.  k <= 128 (`topk` selects more; rows in ascending order or of equal values are slow).  Differentiable in the logits (through `logprob`, `lse`,
    `entropy` and `top_logprobs`), once; see `profk.h` for masked, empty and NaN rows."""
    if isinstance(logits, torch.Tensor) and logits.requires_grad and torch.is_grad_enabled():
        return LogProbs._make(_LogProbsFunction.apply(logits, tokens, k, temperature, bool(entropy)))
    return LogProbs._make((_native or _load()).logprobs(logits, tokens, k, temperature, bool(entropy)))


def logprobs_backward(logits, lse, tokens=None, grad_logprob=None, *, entropy=None, grad_entropy=None, grad_lse=None,
                      top_tokens=None, grad_top=None, lse_rest=None, temperature: float = 1.0):
    """`profk_logprobs_backward_*` on the current stream: the gradient of `logprobs` with respect to the logits, of their
    type, from `lse` (and `lse_rest`, which makes up for its rounding beside large logits; `entropy`, `tokens`, `top_tokens`
    where a gradient refers to them) and upstream gradients."""
    return (_native or _load()).logprobs_backward(logits, lse, lse_rest, tokens, grad_logprob, entropy, grad_entropy, grad_lse,
                                                  top_tokens, grad_top, temperature)


# --- paged cache ----------------------------------------------------------------------------------------------------

class PagesForked(NamedTuple):
    tables: torch.Tensor       # (n, width) int32
    lengths: torch.Tensor      # (n,) int32
    refs: torch.Tensor         # (pages,) int32
    missing: torch.Tensor      # () int32: pages that were needed but not to be had


class PagesCompacted(NamedTuple):
    tables: torch.Tensor       # (n, width) int32
    refs: torch.Tensor         # (pages,) int32
    page_map: torch.Tensor     # (pages,) int32: the new number of each live page, -1 for the others
    live: torch.Tensor         # () int32


def pages_fork(pool, tables, lengths, refs, parents, grow: int = 0, page_size: Optional[int] = None, past_room: bool = False) -> PagesForked:
    """`profk_pages_fork` on the current stream: new sequence i continues old sequence `parents[i]` (a negative number: an
    empty one) with room for `grow` more tokens.  Full pages are shared, a partly filled one stays with the first child and
    is copied for the others, sequences without a child are released.  Copies are made in `pool` ((layers, 2, pages,
    kv_heads, page_size, dim), any strides with dense rows; None with `page_size`: tables and counts only); tables, lengths
    and counts come back new.  tables (n_old, width), lengths (n_old,), refs (pages,), parents (n,): int32.

    A sequence whose table is full gets no longer, and appending to it all the same would write over its last tokens, which its
    siblings share.  Where that can happen, `past_room=True` lets the lengths go on past the table's end, so that
    `pages_append` passes over what has no place."""
    return PagesForked._make((_native or _load()).pages_fork(pool, tables, lengths, refs, parents, grow, -1 if page_size is None else page_size, bool(past_room)))


def pages_compact(pool, tables, refs) -> PagesCompacted:
    """`profk_pages_compact` on the current stream: moves the live pages of `pool` (None: tables and counts only) to its
    front; tables and counts come back new."""
    return PagesCompacted._make((_native or _load()).pages_compact(pool, tables, refs))


def pages_copy(pool, src, dst) -> None:
    """`profk_pages_copy` on the current stream: page src[j] of `pool` to page dst[j], all layers (int32, (n,))."""
    (_native or _load()).pages_copy(pool, src, dst)


def pages_append(k_pages, v_pages, tables, lengths, k, v) -> None:
    """`profk_pages_append` on the current stream: writes `k`, `v` ((seqs, kv_heads, dim), or (seqs, tokens, kv_heads, dim)),
    the keys and values of every sequence's last token(s), to their places in one layer's pages (pages, kv_heads, page_size,
    dim).  `lengths` counts the new tokens already (`pages_fork(grow=...)`; with `past_room=True` where a table may be full);
    tokens behind the table's end or on a page that is not there are passed over."""
    (_native or _load()).pages_append(k_pages, v_pages, tables, lengths, k, v)


def paged_attention(q, k_pages, v_pages, tables, lengths, scale: Optional[float] = None):
    """`profk_paged_attention_*` on the current stream: attention of one new token per sequence over one layer's pages.

    q (seqs, heads, dim), k_pages and v_pages (pages, kv_heads, page_size, dim), bfloat16 or float16, any strides with dense
    rows (a cache laid out tokens first is passed as `.transpose(1, 2)`); tables (seqs, width), lengths (seqs,) int32;
    scale defaults to dim ** -0.5.  The cache is read once for up to 16 query heads to a key.  Returns (out (seqs, heads, dim), lse (seqs, heads) float32)."""
    return (_native or _load()).paged_attention(q, k_pages, v_pages, tables, lengths, scale)


# --- prompts and drafts -----------------------------------------------------------------------------------------------

def rotary_frequencies(dim: int, base: float = 10000.0, stretch: float = 1.0, context: Optional[int] = None, keep: float = 32.0,
                       slow: float = 1.0, device="cuda"):
    """The frequencies of rotary positions over `dim` elements of a head: base ** (-2 i / dim) radians per position, float64.

    For contexts `stretch` times longer than the one a model was trained on: without `context` every frequency is divided by
    `stretch`.  With it (the trained context's length), pairs that make at least `keep` turns over that length keep their
    frequency, those that make at most `slow` are divided by `stretch`, and between the two the share that is divided falls
    linearly with the number of turns.  (Another base is given as such.)"""
    if dim < 2 or dim % 2 != 0 or not base > 0 or not stretch > 0 or (context is not None and not (context > 0 and keep > slow >= 0)):
        import paper_2608_12573_b200 as package

        raise package.ProfkError("rotary_frequencies: dim must be even, base, stretch and context positive, keep above slow")
    f = float(base) ** (-2.0 * torch.arange(dim // 2, dtype=torch.float64) / dim)
    kept = torch.zeros_like(f) if context is None else ((f * context / (2 * math.pi) - slow) / (keep - slow)).clamp(0, 1)
    return (f * kept + f / stretch * (1 - kept)).to(device)


class _RotaryFunction(torch.autograd.Function):
    """Linear in x: the transpose of a turn is the turn by the negative angle, so every derivative is this function again."""
    @staticmethod
    def forward(ctx, x, positions, frequencies, interleaved, magnitude, inverse):
        ctx.save_for_backward(positions, frequencies)
        ctx.how = interleaved, magnitude, inverse
        return _load().rotary(x, positions, frequencies, interleaved, magnitude, inverse)

    @staticmethod
    def backward(ctx, g):
        positions, frequencies = ctx.saved_tensors
        interleaved, magnitude, inverse = ctx.how
        # (an upstream gradient comes in any layout: a broadcast scalar, a permutation)
        if g.dim() > 4 or (g.size(-1) > 1 and g.stride(-1) != 1):
            g = g.contiguous()
        return _RotaryFunction.apply(g, positions, frequencies, interleaved, magnitude, not inverse), None, None, None, None, None


def rotary(x, positions, frequencies, *, interleaved: bool = False, magnitude: float = 1.0, inverse: bool = False):
    """`profk_rotary_*` on the current stream: turns pair i of every head by `positions * frequencies[i]` radians.

    x: CUDA tensor (..., heads, dim), float32, bfloat16 or float16, dense heads, any strides (of more than two leading dimensions:
    evenly spaced on two levels).  positions: int64, broadcast to x's leading dimensions.  frequencies: float64 (pairs,), 2 * pairs <= dim; the rest of a head is left as it is
    (`rotary_frequencies`).  Pairs are elements i and pairs + i, or 2 i and 2 i + 1 with `interleaved`.  `magnitude` scales what
    is turned; `inverse` turns back.  Differentiable in x, any number of times; frequencies that require a gradient are refused."""
    if isinstance(x, torch.Tensor) and x.requires_grad and torch.is_grad_enabled():
        # (grad mode is off in the function's forward, where the call's own check would not see it)
        if isinstance(frequencies, torch.Tensor) and frequencies.requires_grad:
            import paper_2608_12573_b200 as package

            raise package.ProfkError("frequencies requires a gradient, which this call does not have: detach it, or call under torch.no_grad()")
        return _RotaryFunction.apply(x, positions, frequencies, bool(interleaved), magnitude, bool(inverse))
    return (_native or _load()).rotary(x, positions, frequencies, bool(interleaved), magnitude, bool(inverse))


def pages_append_rotary(k_pages, v_pages, tables, lengths, q, k, v, frequencies, *, starts=None, positions=None, interleaved: bool = False,
                        magnitude: float = 1.0):
    """`profk_pages_append_rotary_*` on the current stream: `pages_append` with `rotary` on the way.  Writes the turned keys `k`
    and the values `v` of every sequence's newest tokens to their places in one layer's pages, and returns the turned queries.

    q (None: no queries, returns None), k, v: (seqs, [tokens,] heads or kv_heads, dim), or with `starts` (seqs + 1,) int32 (rows,
    heads or kv_heads, dim), where sequence s has the rows starts[s] to starts[s + 1] - 1, any strides with dense heads; float32,
    bfloat16 or float16, as the pages.  `lengths` counts the new tokens already; a token is turned by its place in its sequence,
    or by `positions` (int64, one per token).  Tokens without a place (see `pages_append`) are turned only; rows that no
    sequence holds come back as zeros."""
    return (_native or _load()).pages_append_rotary(k_pages, v_pages, tables, lengths, q, k, v, frequencies, starts, positions, bool(interleaved), magnitude)


def paged_attention_chunk(q, k_pages, v_pages, tables, lengths, *, starts=None, scale: Optional[float] = None):
    """`profk_paged_attention_chunk_*` on the current stream: attention of several new tokens per sequence (a prompt or a part of it,
    drafted tokens) over one layer's pages, which hold their keys and values already.  Token t of n new ones of a sequence of
    length L sees the tokens up to place L - n + t.

    q: (seqs, tokens, heads, dim), or with `starts` (seqs + 1,) int32 (rows, heads, dim), where sequence s has the rows starts[s] to
    starts[s + 1] - 1; bfloat16 or float16, any strides with dense heads.  Pages, tables, lengths and scale as for
    `paged_attention`, the form for one token.  Returns (out, of q's shape, lse (..., heads) float32); rows that no sequence
    holds come back as 0 and -inf."""
    return (_native or _load()).paged_attention_chunk(q, k_pages, v_pages, tables, lengths, starts, scale)


def adjust_logits(logits, tokens=None, lengths=None, prompts=None, *, repetition=1.0, frequency=0.0, presence=0.0, bias_tokens=None,
                  bias_values=None, mask=None, out=None):
    """`profk_adjust_logits_*` on the current stream: what a sampler lays over logits before `logprobs` or `topk`.

    logits: CUDA tensor (..., V), float32, bfloat16 or float16, dense rows at any stride.  tokens: int64 (..., L), every row's
    prompt and answer, of which the first `lengths` (int32 (...); None: L) count and the first `prompts` of those (int32; None: 0) are
    prompt.  For a token that was seen the logit is divided (if positive, else multiplied) by `repetition`; one that occurs c
    times in the answer loses frequency * c + presence (each a number or a float32 tensor (...)).  Then bias_values (float32 (..., n),
    n <= 8192; time grows with n squared: 300 are cheap, 8192 without a history take milliseconds) are added at bias_tokens (int64), duplicates summed; what `mask` (int32 (..., ceil(V / 32)), bit v % 32 of word
    v // 32: token v is allowed) does not allow becomes -inf.  tokens, biases and mask may be of one dimension, for all rows alike.
    `out` may be `logits`: then only what changes is touched.  Returns the adjusted logits."""
    return (_native or _load()).adjust_logits(logits, tokens, lengths, prompts, repetition, frequency, presence, bias_tokens, bias_values, mask, out)
