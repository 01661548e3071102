"""What autograd may and may not expect of the decoding operators: a derivative that they do not have is refused, not left out."""
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


def test_a_second_derivative_is_refused():
    x = torch.randn(3, 50, device="cuda", requires_grad=True)
    loss = profk.logprobs(x, torch.arange(3, device="cuda")).logprob.sum()
    grad, = torch.autograd.grad(loss, x, create_graph=True)
    plain = torch.log_softmax(x, -1)[torch.arange(3), torch.arange(3)].sum()
    assert (grad - torch.autograd.grad(plain, x)[0]).abs().max() < 1e-5
    with pytest.raises(RuntimeError):
        (loss + (grad ** 2).sum()).backward()              # (a penalty on the gradient: its term would count for nothing)


def _cache():
    pool = torch.randn(1, 2, 6, 2, 16, 64, device="cuda").to(torch.bfloat16)
    tables = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([20, 30], dtype=torch.int32, device="cuda")
    refs = torch.tensor([1, 1, 1, 1, 0, 0], dtype=torch.int32, device="cuda")
    return pool, tables, lengths, refs


def test_tangents_are_refused():
    import torch.autograd.forward_ad as forward

    x, tokens = torch.randn(3, 50, device="cuda"), torch.arange(3, device="cuda")
    r = profk.logprobs(x, tokens, k=2)
    one = torch.ones(3, device="cuda")
    pool, tables, lengths, refs = _cache()
    k, v = pool[0, 0], pool[0, 1]
    q, new = torch.randn(2, 4, 64, device="cuda").to(k.dtype), torch.randn(2, 2, 64, device="cuda").to(k.dtype)
    before = pool.clone()
    with forward.dual_level():
        dual = lambda t: forward.make_dual(t, torch.ones_like(t))  # noqa: E731
        calls = [lambda: profk.logprobs(dual(x), tokens), lambda: profk.logprobs(dual(x.clone().requires_grad_(True)), tokens),
                 lambda: profk.logprobs_backward(dual(x), r.lse, tokens, one), lambda: profk.logprobs_backward(x, r.lse, tokens, dual(one)),
                 lambda: profk.logprobs_backward(x, dual(r.lse), tokens, one), lambda: profk.logprobs_backward(x, r.lse, grad_lse=dual(one)),
                 lambda: profk.paged_attention(dual(q), k, v, tables, lengths), lambda: profk.paged_attention(q, dual(k), v, tables, lengths),
                 lambda: profk.paged_attention(q, k, dual(v), tables, lengths), lambda: profk.pages_append(k, v, tables, lengths, dual(new), new),
                 lambda: profk.pages_append(k, v, tables, lengths, new, dual(new)), lambda: profk.pages_append(dual(k), v, tables, lengths, new, new),
                 lambda: profk.pages_copy(dual(pool), refs[:1], refs[4:5]), lambda: profk.pages_compact(dual(pool), tables, refs),
                 lambda: profk.pages_fork(dual(pool), tables, lengths, refs, refs[:2], grow=1)]
        for n, call in enumerate(calls):
            with pytest.raises(RuntimeError):
                call()
                pytest.fail(f"call {n} was not refused")
        assert torch.equal(profk.logprobs(x, tokens).lse, r.lse)
    assert torch.equal(pool, before)


def test_inputs_that_require_a_gradient_are_refused_in_grad_mode():
    x, tokens = torch.randn(3, 50, device="cuda"), torch.arange(3, device="cuda")
    r = profk.logprobs(x, tokens, k=2)
    one = torch.ones(3, device="cuda")
    pool, tables, lengths, refs = _cache()
    k, v = pool[0, 0], pool[0, 1]
    q, new = torch.randn(2, 4, 64, device="cuda").to(k.dtype), torch.randn(2, 2, 64, device="cuda").to(k.dtype)
    before = pool.clone()
    leaf = lambda t: t.detach().requires_grad_(True)  # noqa: E731
    calls = [lambda: profk.logprobs_backward(leaf(x), r.lse, tokens, one), lambda: profk.logprobs_backward(x, r.lse, tokens, leaf(one)),
             lambda: profk.logprobs_backward(x, leaf(r.lse), tokens, one), lambda: profk.paged_attention(leaf(q), k, v, tables, lengths),
             lambda: profk.paged_attention(q, leaf(k), v, tables, lengths), lambda: profk.paged_attention(q, k, leaf(v), tables, lengths),
             lambda: profk.pages_append(k, v, tables, lengths, leaf(new), new), lambda: profk.pages_append(k, v, tables, lengths, new, leaf(new)),
             lambda: profk.pages_append(leaf(k), v, tables, lengths, new, new), lambda: profk.pages_copy(leaf(pool), refs[:1], refs[4:5]),
             lambda: profk.pages_compact(leaf(pool), tables, refs), lambda: profk.pages_fork(leaf(pool), tables, lengths, refs, refs[:2], grow=1)]
    for n, call in enumerate(calls):
        with pytest.raises(profk.ProfkError):
            call()
            pytest.fail(f"call {n} was not refused")
    assert torch.equal(pool, before)
    want = profk.paged_attention(q, k, v, tables, lengths)
    with torch.no_grad():
        got = profk.paged_attention(leaf(q), k, v, tables, lengths)
        profk.logprobs_backward(leaf(x), r.lse, tokens, one)
    assert torch.equal(got[0], want[0])


def test_writes_to_a_cache_are_seen_by_autograd():
    pool, tables, lengths, refs = _cache()
    new = torch.randn(2, 2, 64, device="cuda").to(pool.dtype)
    k, v = pool[0, 0], pool[0, 1]
    calls = [lambda: profk.pages_append(k, v, tables, lengths, new, new), lambda: profk.pages_copy(pool, refs[4:5], refs[:1]),
             lambda: profk.pages_fork(pool, tables, lengths, refs, torch.zeros(2, dtype=torch.int32, device="cuda"), grow=1), lambda: profk.pages_compact(pool, tables, refs)]
    for n, call in enumerate(calls):
        weight = torch.ones((), device="cuda", dtype=pool.dtype, requires_grad=True)
        kept = weight * k                                        # autograd keeps a view of the cache for the weight's gradient
        call()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            kept.sum().backward()
            pytest.fail(f"call {n} was not noticed")
    with torch.inference_mode():
        other = pool.clone()
        profk.pages_append(other[0, 0], other[0, 1], tables, lengths, new, new)
    with torch.no_grad():                                        # an inference tensor outside of inference mode
        profk.pages_append(other[0, 0], other[0, 1], tables, lengths, new, new)
