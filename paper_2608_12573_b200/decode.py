"""The operators around a selection in a decoding loop: log probabilities with entropy and top alternatives (and their
gradient).  Like the rest of the binding, these functions only marshal arguments into the C ABI; nothing is synchronised.
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
    f32 = torch.float32
    _call(fn, dev, x.data_ptr(), rows, vocab, stride, float(temperature), _of_row(lse, "lse", f32, lead, dev),
          _of_row(lse_rest, "lse_rest", f32, lead, dev),
          _of_row(tokens, "tokens", torch.int64, lead, dev), _of_row(grad_logprob, "grad_logprob", f32, lead, dev),
          _of_row(entropy, "entropy", f32, lead, dev), _of_row(grad_entropy, "grad_entropy", f32, lead, dev),
          _of_row(grad_lse, "grad_lse", f32, lead, dev), k,
          _of_row(top_tokens, "top_tokens", torch.int64, (*lead, k), dev) if k else None,
          _of_row(grad_top, "grad_top", f32, (*lead, k), dev) if k else None, _stream(dev), grad.data_ptr(), vocab)
    return grad
