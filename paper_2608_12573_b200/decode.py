"""The operators around a selection in a decoding loop: log probabilities with entropy and top alternatives (and their
gradient), the forking and compaction of the pages of a key-value cache, and attention of one token over them.  Like the rest of the binding, these functions only marshal arguments into the C ABI; nothing is synchronised.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

import paper_2608_12573_b200 as _profk

_P, _I, _D = ctypes.c_void_p, ctypes.c_int64, ctypes.c_double
_SUFFIX = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16"}
_SIGNATURES = {
    "logprobs": [_P, _I, _I, _I, _P, _I, _D, _P, _P, _P, _P, _P, _P, _P],
    "logprobs_backward": [_P, _I, _I, _I, _D, _P, _P, _P, _P, _P, _P, _P, _I, _P, _P, _P, _P, _I],
}
_INT, _F32 = torch.int32, torch.float32


class _Pool(ctypes.Structure):
    _fields_ = [("base", _P)] + [(n, _I) for n in ("layers", "kv_heads", "page_size", "row_bytes", "layer", "kv", "page", "head", "token")]


class _PageStrides(ctypes.Structure):
    _fields_ = [("page", _I), ("head", _I), ("token", _I)]


_POOL, _STRIDES, _BYTES, _THREE = ctypes.POINTER(_Pool), ctypes.POINTER(_PageStrides), ctypes.POINTER(ctypes.c_size_t), ctypes.POINTER(_I * 3)
_SIGNATURES.update({
    "paged_attention_workspace_bytes": [_I, _BYTES],
    "paged_attention": [_P, _I, _I, _P, _P, _STRIDES, _STRIDES, _P, _I, _P, _I, _I, _I, _I, _I, _I, _I, _D, _P, ctypes.c_size_t, _P, _P, _P],
    "pages_fork_workspace_bytes": [_I, _I, _I, _I, _I, _BYTES],
    "pages_fork": [_POOL, _P, _I, _I, _I, _P, _P, _I, _P, _I, _I, _I, _P, ctypes.c_size_t, _P, _P, _P, _P, _P],
    "pages_compact_workspace_bytes": [_I, _BYTES],
    "pages_compact": [_POOL, _P, _I, _I, _I, _P, _I, _P, ctypes.c_size_t, _P, _P, _P, _P, _P],
    "pages_copy": [_POOL, _I, _P, _P, _I, _P],
    "pages_append": [_P, _P, _THREE, _THREE, _P, _P, _STRIDES, _STRIDES, _P, _I, _P, _I, _I, _I, _I, _I, _I, _I, _P],
})
_functions: dict = {}


def _function(name: str, dtype):
    """The entry point `profk_<name>_<dtype>` (`profk_<name>` for dtype None), with its argument types declared."""
    fn = _functions.get((name, dtype))
    if fn is None:
        if dtype is not None and dtype not in _SUFFIX:
            raise _profk.ProfkError(f"unsupported dtype {dtype}: float32, bfloat16 and float16 only")
        fn = getattr(_profk.lib(), f"profk_{name}" if dtype is None else f"profk_{name}_{_SUFFIX[dtype]}")
        fn.argtypes = _SIGNATURES[name]
        _functions[(name, dtype)] = fn
    return fn


def _call(fn, device, *args) -> None:
    """Calls `fn` with the tensors' device current (the library launches on the current device)."""
    if device.index == torch.cuda.current_device():
        code = fn(*args)
    else:
        with torch.cuda.device(device):
            code = fn(*args)
    if code:
        _profk._check(code, fn.__name__)


def _stream(device) -> int:
    return torch.cuda.current_stream(device).cuda_stream


def _cuda(x, what: str):
    if not x.is_cuda:
        raise _profk.ProfkError(f"{what} must be a CUDA tensor")
    return x


def _of_row(x, what: str, dtype, shape, device):
    """The data pointer of an optional per-row tensor, or None."""
    if x is None:
        return None
    if x.dtype != dtype or x.shape != shape or x.device != device or not x.is_contiguous():
        raise _profk.ProfkError(f"{what} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}")
    return x.data_ptr()


class LogProbs(NamedTuple):
    """What `logprobs` returns; all but the tokens are float32.  A part that was not asked for is None."""
    logprob: Optional[torch.Tensor]         # (...)    of the given tokens
    lse: torch.Tensor                       # (...)    ln sum e^(logit / temperature)
    entropy: Optional[torch.Tensor]         # (...)
    top_logprobs: Optional[torch.Tensor]    # (..., k)
    top_tokens: Optional[torch.Tensor]      # (..., k) int64
    lse_rest: torch.Tensor                  # (...)    what the rounding of lse left off, for `logprobs_backward`


def _matrix(x, what: str):
    """(rows, V) view of a (..., V) tensor whose rows are dense and evenly spaced."""
    _cuda(x, what)
    if x.dim() < 1 or x.shape[-1] < 1 or x.numel() == 0:
        raise _profk.ProfkError(f"{what} must have at least one row and one column")
    if x.dim() != 2:
        try:
            x = x.view(-1, x.shape[-1])
        except RuntimeError:
            raise _profk.ProfkError(f"{what}: the leading dimensions must be evenly spaced") from None
    if x.shape[1] > 1 and x.stride(1) != 1 or x.shape[0] > 1 and x.stride(0) < x.shape[1]:
        raise _profk.ProfkError(f"{what} must have dense rows that do not overlap")
    return x


def _forward(logits, tokens, k, temperature, entropy) -> LogProbs:
    x = _matrix(logits, "logits")
    rows, vocab = x.shape
    dev, lead = x.device, logits.shape[:-1]
    fn = _function("logprobs", x.dtype)
    tok = _of_row(tokens, "tokens", torch.int64, lead, dev)
    lse = torch.empty(lead, dtype=torch.float32, device=dev)
    rest = torch.empty_like(lse)
    logprob = torch.empty_like(lse) if tok is not None else None
    ent = torch.empty_like(lse) if entropy else None
    top_lp = torch.empty((*lead, k), dtype=torch.float32, device=dev) if k > 0 else None
    top_tok = torch.empty((*lead, k), dtype=torch.int64, device=dev) if k > 0 else None
    _call(fn, dev, x.data_ptr(), rows, vocab, x.stride(0) if rows > 1 else vocab, tok, k, temperature, _stream(dev),
          None if logprob is None else logprob.data_ptr(), lse.data_ptr(), rest.data_ptr(), None if ent is None else ent.data_ptr(),
          None if top_lp is None else top_lp.data_ptr(), None if top_tok is None else top_tok.data_ptr())
    return LogProbs(logprob, lse, ent, top_lp, top_tok, rest)


class _LogProbsFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, k, temperature, entropy):
        r = _forward(logits, tokens, k, temperature, entropy)
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

        grad = logprobs_backward(logits, lse, tokens, dense(g_logprob), entropy=entropy, grad_entropy=dense(g_entropy),
                                 grad_lse=dense(g_lse), top_tokens=top, grad_top=dense(g_top), lse_rest=rest,
                                 temperature=ctx.temperature)
        return grad, None, None, None, None


def logprobs(logits, tokens=None, k: int = 0, temperature: float = 1.0, entropy: bool = True) -> LogProbs:
    """`profk_logprobs_*` on the current stream: log probabilities of `tokens`, log-sum-exp, entropy and the `k` most
    probable tokens of every row of `logits / temperature`, in one read of the logits.

    logits: CUDA tensor (..., V), float32, bfloat16 or float16, dense rows at any stride.  tokens: int64 (...), negative
    where no token is given.  k <= 128 (`topk` selects more).  Differentiable in the logits (through `logprob`, `lse`,
    `entropy` and `top_logprobs`); see `profk.h` for masked, empty and NaN rows."""
    if logits.requires_grad and torch.is_grad_enabled():
        return LogProbs(*_LogProbsFunction.apply(logits, tokens, int(k), float(temperature), bool(entropy)))
    return _forward(logits, tokens, int(k), float(temperature), bool(entropy))


def logprobs_backward(logits, lse, tokens=None, grad_logprob=None, *, entropy=None, grad_entropy=None, grad_lse=None,
                      top_tokens=None, grad_top=None, lse_rest=None, temperature: float = 1.0):
    """`profk_logprobs_backward_*` on the current stream: the gradient of `logprobs` with respect to the logits, of their
    type, from `lse` (and `lse_rest`, which makes up for its rounding beside large logits; `entropy`, `tokens`, `top_tokens`
    where a gradient refers to them) and upstream gradients."""
    x = _matrix(logits, "logits")
    rows, vocab = x.shape
    dev, lead = x.device, logits.shape[:-1]
    fn = _function("logprobs_backward", x.dtype)
    k = 0
    if grad_top is not None:
        if top_tokens is None:
            raise _profk.ProfkError("grad_top needs top_tokens")
        k = top_tokens.shape[-1]
    stride = x.stride(0) if rows > 1 else vocab
    grad = torch.empty(logits.shape, dtype=x.dtype, device=dev)
    f32 = _F32
    _call(fn, dev, x.data_ptr(), rows, vocab, stride, float(temperature), _of_row(lse, "lse", f32, lead, dev),
          _of_row(lse_rest, "lse_rest", f32, lead, dev),
          _of_row(tokens, "tokens", torch.int64, lead, dev), _of_row(grad_logprob, "grad_logprob", f32, lead, dev),
          _of_row(entropy, "entropy", f32, lead, dev), _of_row(grad_entropy, "grad_entropy", f32, lead, dev),
          _of_row(grad_lse, "grad_lse", f32, lead, dev), k,
          _of_row(top_tokens, "top_tokens", torch.int64, (*lead, k), dev) if k else None,
          _of_row(grad_top, "grad_top", f32, (*lead, k), dev) if k else None, _stream(dev), grad.data_ptr(), vocab)
    return grad


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


_workspace_sizes: dict = {}


def _workspace(name: str, device, *sizes):
    """Scratch for one call: a torch allocation on the current stream, so that calls on several streams do not meet."""
    key = (name, device.index, *sizes)
    need = _workspace_sizes.get(key)
    if need is None:
        n = ctypes.c_size_t()
        _call(_function(name, None), device, *sizes, ctypes.byref(n))
        if len(_workspace_sizes) > 4096:
            _workspace_sizes.clear()
        need = _workspace_sizes[key] = int(n.value)
    return torch.empty(need, dtype=torch.uint8, device=device), need


def _ints(x, what: str, dims: int, device):
    """An int32 tensor of `dims` dimensions on `device` with a dense last one (one-dimensional: contiguous)."""
    if not x.is_cuda or x.dtype != _INT or x.dim() != dims or x.device != device or \
            x.numel() > 0 and x.shape[-1] > 1 and x.stride(-1) != 1:
        raise _profk.ProfkError(f"{what} must be a dense int32 tensor of {dims} dimension(s) on {device}")
    return x


def _tables(tables, device):
    _ints(tables, "tables", 2, device)
    if tables.shape[1] < 1 or tables.shape[0] > 1 and tables.stride(0) < tables.shape[1]:
        raise _profk.ProfkError("tables must have rows of at least one entry that do not overlap")
    return tables.stride(0) if tables.shape[0] > 1 else tables.shape[1]


def _pool_of(pool):
    """The C description of a cache tensor (layers, 2, pages, kv_heads, page_size, dim); dense rows, other strides any."""
    _cuda(pool, "pool")
    if pool.dim() != 6 or pool.shape[1] != 2 or pool.numel() == 0:
        raise _profk.ProfkError("pool must be of shape (layers, 2, pages, kv_heads, page_size, dim)")
    if pool.shape[5] > 1 and pool.stride(5) != 1:
        raise _profk.ProfkError("pool must have dense rows")
    size = pool.element_size()
    return _Pool(pool.data_ptr(), pool.shape[0], pool.shape[3], pool.shape[4], pool.shape[5] * size, *(s * size for s in pool.stride()[:5]))


def pages_fork(pool, tables, lengths, refs, parents, grow: int = 0, page_size: Optional[int] = None) -> PagesForked:
    """`profk_pages_fork` on the current stream: new sequence i continues old sequence `parents[i]` (a negative number: an
    empty one) with room for `grow` more tokens.  Full pages are shared, a partly filled one stays with the first child and
    is copied for the others, sequences without a child are released.  Copies are made in `pool` ((layers, 2, pages,
    kv_heads, page_size, dim), any strides with dense rows; None with `page_size`: tables and counts only); tables, lengths
    and counts come back new.  tables (n_old, width), lengths (n_old,), refs (pages,), parents (n,): int32."""
    dev = _cuda(refs, "refs").device
    _ints(refs, "refs", 1, dev), _ints(lengths, "lengths", 1, dev), _ints(parents, "parents", 1, dev)
    stride = _tables(tables, dev)
    n_old, width = tables.shape
    n, pages = parents.shape[0], refs.shape[0]
    if lengths.shape[0] != n_old:
        raise _profk.ProfkError("tables and lengths must have the same number of sequences")
    if pool is not None:
        desc = ctypes.byref(_pool_of(pool))
        if pool.device != dev or pool.shape[2] != pages or page_size not in (None, pool.shape[4]):
            raise _profk.ProfkError("pool must hold as many pages as refs counts, of page_size tokens, on the same device")
        page_size = pool.shape[4]
    else:
        desc = None
        if page_size is None:
            raise _profk.ProfkError("without a pool the page_size must be given")
    ws, need = _workspace("pages_fork_workspace_bytes", dev, n_old, n, pages, page_size, grow)
    new_tables = torch.empty((n, width), dtype=_INT, device=dev)
    new_lengths = torch.empty(n, dtype=_INT, device=dev)
    new_refs = torch.empty_like(refs)
    missing = torch.empty((), dtype=_INT, device=dev)
    _call(_function("pages_fork", None), dev, desc, tables.data_ptr(), n_old, width, stride, lengths.data_ptr(), refs.data_ptr(), pages,
          parents.data_ptr(), n, page_size, grow, ws.data_ptr(), need, _stream(dev), new_tables.data_ptr(), new_lengths.data_ptr(),
          new_refs.data_ptr(), missing.data_ptr())
    return PagesForked(new_tables, new_lengths, new_refs, missing)


def pages_compact(pool, tables, refs) -> PagesCompacted:
    """`profk_pages_compact` on the current stream: moves the live pages of `pool` (None: tables and counts only) to its
    front; tables and counts come back new."""
    dev = _cuda(refs, "refs").device
    _ints(refs, "refs", 1, dev)
    stride = _tables(tables, dev)
    n, width = tables.shape
    pages = refs.shape[0]
    desc = None
    if pool is not None:
        desc = ctypes.byref(_pool_of(pool))
        if pool.device != dev or pool.shape[2] != pages:
            raise _profk.ProfkError("pool must hold as many pages as refs counts, on the same device")
    ws, need = _workspace("pages_compact_workspace_bytes", dev, pages)
    new_tables = torch.empty((n, width), dtype=_INT, device=dev)
    new_refs, page_map = torch.empty_like(refs), torch.empty_like(refs)
    live = torch.empty((), dtype=_INT, device=dev)
    _call(_function("pages_compact", None), dev, desc, tables.data_ptr(), n, width, stride, refs.data_ptr(), pages, ws.data_ptr(), need,
          _stream(dev), new_tables.data_ptr(), new_refs.data_ptr(), page_map.data_ptr(), live.data_ptr())
    return PagesCompacted(new_tables, new_refs, page_map, live)


def pages_copy(pool, src, dst) -> None:
    """`profk_pages_copy` on the current stream: page src[j] of `pool` to page dst[j], all layers (int32, (n,))."""
    desc = _pool_of(pool)
    _ints(src, "src", 1, pool.device), _ints(dst, "dst", 1, pool.device)
    if src.shape != dst.shape:
        raise _profk.ProfkError("src and dst must have the same length")
    _call(_function("pages_copy", None), pool.device, ctypes.byref(desc), pool.shape[2], src.data_ptr(), dst.data_ptr(), src.shape[0],
          _stream(pool.device))


def _pages_pair(k_pages, v_pages):
    """Checks one layer's keys and values (pages, kv_heads, page_size, dim)."""
    _cuda(k_pages, "k_pages")
    if k_pages.dim() != 4 or k_pages.shape != v_pages.shape or k_pages.dtype != v_pages.dtype or k_pages.device != v_pages.device or k_pages.numel() == 0:
        raise _profk.ProfkError("k_pages and v_pages must be alike, of shape (pages, kv_heads, page_size, dim)")
    if k_pages.shape[3] > 1 and not k_pages.stride(3) == v_pages.stride(3) == 1:
        raise _profk.ProfkError("k_pages and v_pages must have dense rows")


def pages_append(k_pages, v_pages, tables, lengths, k, v) -> None:
    """`profk_pages_append` on the current stream: writes `k`, `v` ((seqs, kv_heads, dim), or (seqs, tokens, kv_heads, dim)),
    the keys and values of every sequence's last token(s), to their places in one layer's pages (pages, kv_heads, page_size,
    dim).  `lengths` counts the new tokens already (`pages_fork(grow=...)`)."""
    _pages_pair(k_pages, v_pages)
    dev = k_pages.device
    stride = _tables(tables, dev)
    _ints(lengths, "lengths", 1, dev)
    k, v = (x.unsqueeze(1) if x.dim() == 3 else x for x in (k, v))
    pages, kv_heads, page_size, dim = k_pages.shape
    seqs, width = tables.shape
    if k.shape != v.shape or k.dim() != 4 or k.shape[0] != seqs or k.shape[2:] != (kv_heads, dim) or lengths.shape[0] != seqs:
        raise _profk.ProfkError("k and v must be of shape (seqs, [tokens,] kv_heads, dim), one sequence per row of the tables")
    if not k.dtype == v.dtype == k_pages.dtype or not k.device == v.device == dev or dim > 1 and not k.stride(3) == v.stride(3) == 1:
        raise _profk.ProfkError("k and v must have the pages' type and device, and dense rows")
    size = k.element_size()
    three = [(_I * 3)(*(s * size for s in x.stride()[:3])) for x in (k, v)]
    at = [_PageStrides(*(s * size for s in x.stride()[:3])) for x in (k_pages, v_pages)]
    _call(_function("pages_append", None), dev, k.data_ptr(), v.data_ptr(), ctypes.byref(three[0]), ctypes.byref(three[1]), k_pages.data_ptr(),
          v_pages.data_ptr(), ctypes.byref(at[0]), ctypes.byref(at[1]), tables.data_ptr(), stride, lengths.data_ptr(), seqs, k.shape[1], kv_heads,
          dim * size, page_size, pages, width, _stream(dev))


def paged_attention(q, k_pages, v_pages, tables, lengths, scale: Optional[float] = None):
    """`profk_paged_attention_*` on the current stream: attention of one new token per sequence over one layer's pages.

    q (seqs, heads, dim), k_pages and v_pages (pages, kv_heads, page_size, dim), bfloat16 or float16, any strides with dense
    rows (a cache laid out tokens first is passed as `.transpose(1, 2)`); tables (seqs, width), lengths (seqs,) int32;
    scale defaults to dim ** -0.5.  Returns (out (seqs, heads, dim), lse (seqs, heads) float32)."""
    _cuda(q, "q")
    _pages_pair(k_pages, v_pages)
    dev, dtype = q.device, q.dtype
    if q.dim() != 3 or q.numel() == 0 or q.shape[2] > 1 and q.stride(2) != 1:
        raise _profk.ProfkError("q must be of shape (seqs, heads, dim) with dense rows")
    seqs, heads, dim = q.shape
    pages, kv_heads, page_size, _ = k_pages.shape
    stride = _tables(tables, dev)
    _ints(lengths, "lengths", 1, dev)
    if k_pages.dtype != dtype or k_pages.device != dev or k_pages.shape[3] != dim or heads % kv_heads or tables.shape[0] != seqs or lengths.shape[0] != seqs:
        raise _profk.ProfkError("q, pages, tables and lengths do not belong together (type, device, dim, heads or sequences differ)")
    if dtype not in (torch.bfloat16, torch.float16):
        raise _profk.ProfkError(f"unsupported dtype {dtype}: bfloat16 and float16 only")
    ws, need = _workspace("paged_attention_workspace_bytes", dev, dim)
    out = torch.empty((seqs, heads, dim), dtype=dtype, device=dev)
    lse = torch.empty((seqs, heads), dtype=_F32, device=dev)
    _call(_function("paged_attention", dtype), dev, q.data_ptr(), q.stride(0), q.stride(1), k_pages.data_ptr(), v_pages.data_ptr(),
          ctypes.byref(_PageStrides(*k_pages.stride()[:3])), ctypes.byref(_PageStrides(*v_pages.stride()[:3])), tables.data_ptr(), stride,
          lengths.data_ptr(), seqs, heads, kv_heads, dim, page_size, pages, tables.shape[1], dim ** -0.5 if scale is None else scale,
          ws.data_ptr(), need, _stream(dev), out.data_ptr(), lse.data_ptr())
    return out, lse
