"""Log probabilities and their gradient where sizes, values and buffers reach the limits of what is accepted."""
import ctypes

import pytest
import torch

import paper_2608_12573_b200 as profk
from paper_2608_12573_b200 import _build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    _build.build()
    profk.lib()
    torch.cuda.set_device(0)


def test_as_many_rows_as_are_accepted():
    """2^31 - 1 rows of one logit: a row's number and the step to the next one together pass 31 bits.  Of one logit the
    log-sum-exp is the logit itself, exactly."""
    rows = 2 ** 31 - 1
    x = torch.empty(rows, 1, dtype=torch.float16, device="cuda")
    step = 1 << 27
    for r in range(0, rows, step):
        n = min(step, rows - r)
        x[r:r + n, 0] = ((torch.arange(r, r + n, device="cuda") * 7919) % 4096 - 2048).half()
    lse = profk.logprobs(x, entropy=False).lse
    for r in range(0, rows, step):
        assert torch.equal(lse[r:r + step], x[r:r + step, 0].float())


# --- gradient in place of the logits ---------------------------------------------------------------------------------

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _backward(x, grad, lse, rest=None, tokens=None, g_logprob=None, entropy=None, g_entropy=None, g_lse=None, top=None, g_top=None):
    """The C call on (rows, V) tensors of any row stride; its status."""
    at = lambda t: ctypes.c_void_p(None if t is None else t.data_ptr())  # noqa: E731
    call = getattr(profk.lib(), "profk_logprobs_backward_" + {d: n for n, d in DTYPES.items()}[x.dtype])
    rows, vocab = x.shape
    return call(at(x), ctypes.c_int64(rows), ctypes.c_int64(vocab), ctypes.c_int64(x.stride(0)), ctypes.c_double(1.0), at(lse), at(rest), at(tokens),
                at(g_logprob), at(entropy), at(g_entropy), at(g_lse), ctypes.c_int64(0 if top is None else top.shape[1]), at(top), at(g_top),
                ctypes.c_void_p(torch.cuda.current_stream().cuda_stream), at(grad), ctypes.c_int64(grad.stride(0)))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("vocab,pad", [(1, 0), (7, 1), (5003, 0), (40000, 24)])
def test_gradient_in_place_of_the_logits(dtype, vocab, pad):
    """Allowed where no entry is picked out; the tokens and alternatives of the forward call may be there all the same.  The
    same bits as in rows of their own."""
    x = (torch.randn(9, vocab + pad, device="cuda") * 3).to(DTYPES[dtype])[:, :vocab]
    k = min(3, vocab)
    r = profk.logprobs(x, torch.arange(9, device="cuda") % vocab, k=k)
    up = torch.randn(2, 9, device="cuda")
    args = dict(rest=r.lse_rest, tokens=torch.arange(9, device="cuda") % vocab, entropy=r.entropy, g_entropy=up[0].contiguous(), g_lse=up[1].contiguous(), top=r.top_tokens)
    want = torch.empty_like(x)
    assert _backward(x, want, r.lse, **args) == 0
    assert _backward(x, x, r.lse, **args) == 0
    assert torch.equal(x, want)


# --- logits at the ends of fp32's range ------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("temperature", [0.7, 0.5])
def test_rows_whose_scaled_logits_pass_the_range(dtype, temperature):
    """Largest logits of the type's lowest and largest values at temperatures below 1: lse is infinite, log probabilities and
    entropy are those of the tied tokens, the gradient is zero."""
    import math

    vocab, info = 3001, torch.finfo(DTYPES[dtype])
    x = torch.full((4, vocab), info.min, dtype=DTYPES[dtype], device="cuda")
    x[1, 7:] = -float("inf")                           # seven of them
    x[2] = 0.0
    x[2, 5:10] = info.max                              # five of the largest value
    x[3] = torch.randn(vocab, device="cuda")           # an ordinary row beside them
    tokens = torch.tensor([3, 2, 6, 11], device="cuda")
    r = profk.logprobs(x, tokens, k=4, temperature=temperature)
    assert r.lse[:3].tolist() == [-float("inf"), -float("inf"), float("inf")] and torch.isfinite(r.lse[3])
    want = torch.tensor([-math.log(n) for n in (vocab, 7, 5)], device="cuda")
    assert (r.logprob[:3] - want).abs().max() < 1e-5 and (r.entropy[:3] + want).abs().max() < 1e-5
    assert (r.top_logprobs[:3] - want[:, None]).abs().max() < 1e-5
    assert r.top_tokens.tolist()[:3] == [[0, 1, 2, 3], [0, 1, 2, 3], [5, 6, 7, 8]]
    one = torch.ones(4, device="cuda")
    grad = profk.logprobs_backward(x, r.lse, tokens, one, entropy=r.entropy, grad_entropy=one, grad_lse=one, top_tokens=r.top_tokens,
                                   grad_top=torch.ones(4, 4, device="cuda"), lse_rest=r.lse_rest, temperature=temperature)
    assert (grad[:3] == 0).all() and (grad[3] != 0).any() and torch.isfinite(grad[3]).all()


# --- alternatives that are none --------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("k", [1, 3, 128])
def test_gradient_of_places_without_a_token(dtype, k):
    """A list of alternatives that is filled up with -1 (or names tokens outside the vocabulary): the same bits as with
    gradients of zero there."""
    vocab = 517
    x = torch.randn(5, vocab, device="cuda").to(DTYPES[dtype])
    r = profk.logprobs(x, k=k)
    top, g_top = r.top_tokens.clone(), torch.randn(5, k, device="cuda")
    none = torch.rand(5, k, device="cuda") < 0.4
    none[0], none[1] = True, False
    top[none] = -1
    top[2][none[2]] = vocab
    top[3][none[3]] = 1 << 40
    zeroed = torch.where(none, torch.zeros_like(g_top), g_top)
    got = profk.logprobs_backward(x, r.lse, top_tokens=top, grad_top=g_top, lse_rest=r.lse_rest)
    want = profk.logprobs_backward(x, r.lse, top_tokens=r.top_tokens, grad_top=zeroed, lse_rest=r.lse_rest)
    assert torch.equal(got, want) and (got[0] == 0).all() and (got[1] != 0).any()


# --- logits far from zero --------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("temperature", [1.0, 1.3, 5.0, 0.9999])
@pytest.mark.parametrize("offset", [0, 1])
def test_gradient_of_logits_far_from_zero(dtype, temperature, offset):
    """Rows whose largest logits are large and tied: the gradient is that of the tied tokens, at any temperature.  Log
    probabilities are exact to 2^-22 of themselves here (ln s to three bits less than a float), 12 * 2^-20 at most, and the
    logits' differences times 1 / temperature to 2^-23 of themselves: 2e-5 of a probability's part, with the entropy's factor of
    12 besides; and half a unit in the last place."""
    vocab, info = 5003, torch.finfo(DTYPES[dtype])
    values = [v for v in (info.min, info.max, -1e30, 3e20, -1e12, 2.5e9, -1.3e9, 9e8, -6e4, 2e3) if info.min <= v <= info.max]
    if temperature < 1:
        values = [v for v in values if abs(v) < 1e38]
    x = torch.empty(len(values), vocab + 1, dtype=DTYPES[dtype], device="cuda")[:, offset:offset + vocab]
    for row, v in enumerate(values):
        x[row] = v                                            # everything tied, then a part of it masked or below
        x[row, 100 + 400 * row:] = -float("inf") if row % 2 or v == info.min else v - abs(v) * 2.0 ** -6
        x[row, 7:40:3] = -float("inf")
    rows = len(values)
    tokens = torch.arange(rows, device="cuda")
    up = torch.randn(3, rows, device="cuda")
    k = 3
    g_top = torch.randn(rows, k, device="cuda")
    r = profk.logprobs(x, tokens, k=k, temperature=temperature)
    args = dict(entropy=r.entropy, grad_entropy=up[1].contiguous(), grad_lse=up[2].contiguous(), top_tokens=r.top_tokens, grad_top=g_top, lse_rest=r.lse_rest,
                temperature=temperature)
    got = profk.logprobs_backward(x, r.lse, tokens, up[0].contiguous(), **args).double()
    z = x.double() / temperature
    d = z - z.amax(1, keepdim=True)
    logp = d - torch.exp(d).sum(1, keepdim=True).log()
    p = torch.exp(logp)
    entropy = torch.special.entr(p).sum(1, keepdim=True)
    one = torch.zeros_like(z)
    one[tokens, tokens] += up[0].double()
    one.scatter_add_(1, r.top_tokens, g_top.double())
    inner = one.sum(1, keepdim=True) - up[2].double()[:, None]
    safe = torch.where(p > 0, logp, 0.0)
    want = (one - p * (inner + up[1].double()[:, None] * (safe + entropy))) / temperature
    size = p * (up[0].abs() + up[2].abs() + g_top.abs().sum(1) + 12 * up[1].abs()).double()[:, None] / temperature
    allowed = 2e-5 * size + 2.0 ** -22 * want.abs() + 0.5 * info.eps * want.abs() + (2.0 ** -25 if dtype == "f16" else 1e-38)
    assert ((got - want).abs() <= allowed).all(), ((got - want).abs() - allowed).amax(1)
    if temperature == 1.0:                                    # in place of the logits, without picked entries
        args = dict(rest=r.lse_rest, entropy=r.entropy, g_entropy=up[1].contiguous(), g_lse=up[2].contiguous())
        out = torch.empty(rows, vocab + 1, dtype=x.dtype, device="cuda")[:, offset:offset + vocab]
        assert _backward(x, out, r.lse, **args) == 0 and _backward(x, x, r.lse, **args) == 0
        assert torch.equal(x, out)


def test_gradient_of_neighbouring_logits_far_from_zero():
    """Two fp32 logits that differ in their last bit, 1e13 from zero: the smaller one's probability is 0, whatever the
    temperature rounds their quotients to."""
    rng = torch.Generator().manual_seed(5)
    rows, vocab = 400, 33
    big = (torch.rand(rows, generator=rng) + 1) * 2.0 ** torch.randint(40, 120, (rows,), generator=rng)
    big = torch.where(torch.rand(rows, generator=rng) < 0.5, big, -big)
    x = torch.full((rows, vocab), -float("inf"))
    x[:, 3], x[:, 20] = big, torch.nextafter(big, torch.full_like(big, -float("inf")))
    x[:, 30] = big
    x = x.cuda()
    g = torch.ones(rows, device="cuda")
    for temperature in (1.1, 1.7, 3.0, 0.77):
        r = profk.logprobs(x, temperature=temperature)
        got = profk.logprobs_backward(x, r.lse, grad_lse=g, lse_rest=r.lse_rest, temperature=temperature)       # the probabilities / temperature
        want = torch.zeros(rows, vocab, device="cuda")
        want[:, [3, 30]] = 0.5 / temperature
        assert (got - want).abs().max() < 1e-5
