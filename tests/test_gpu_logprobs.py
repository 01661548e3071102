"""Log probabilities, entropy and top alternatives, and their gradient, against the 64-bit oracle on a GPU.

Tolerances.  A probability e^(z - m) is taken as 2^y, y = (x - max) log2(e) / T, with two roundings of y (2^-23 |y|) and
one of the exponential (2^-22), and a row's sum is joined from parts of at most a few hundred terms (2^-24 each, 2^-16 in
all at worst).  With |y| <= 64 where p matters that is 2^-17 + 2^-16 < 3e-5 of s at worst, so ln s and with it lse and the log
probabilities are held to 3e-5 absolute plus 2^-22 of the value; the entropy, whose terms carry |ln p| <= 45 more, to 1e-4
plus 2^-20 of the value.  Gradients: see `logprobs_gradient_row`, whose bound is taken four times, plus half a unit in the
last place of the output type (and its smallest step)."""
import numpy as np
import pytest
import torch

import paper_2608_12573_b200 as profk
from oracle import decode as oracle
from paper_2608_12573_b200 import _build

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
STEP = {name: (torch.finfo(d).eps, torch.finfo(d).smallest_normal if name != "f16" else 2.0 ** -24) for name, d in DTYPES.items()}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    _build.build()
    profk.lib()
    torch.cuda.set_device(0)


def _near(got, want, atol, rtol, what):
    got = np.asarray(got, dtype=np.float64)
    want = np.asarray(want, dtype=np.float64)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    finite = np.isfinite(want)
    ok = same | (finite & np.isfinite(got) & (np.abs(got - np.where(finite, want, 0)) <= atol + rtol * np.abs(np.where(finite, want, 0))))
    assert ok.all(), f"{what}: {got[~ok][:4]} instead of {want[~ok][:4]}"


def _check(x, tokens, k, temperature, entropy=True):
    r = profk.logprobs(x, tokens, k=k, temperature=temperature, entropy=entropy)
    torch.cuda.synchronize()
    host, tok = x.float().cpu().numpy(), tokens.cpu().numpy()
    want = [oracle.logprobs_row(host[i], int(tok[i]), k, temperature) for i in range(host.shape[0])]
    _near(r.lse.cpu(), [w["lse"] for w in want], 3e-5, 2.0 ** -22, "lse")
    _near(r.logprob.cpu(), [w["logprob"] for w in want], 3e-5, 2.0 ** -22, "logprob")
    if entropy:
        _near(r.entropy.cpu(), [w["entropy"] for w in want], 1e-4, 2.0 ** -20, "entropy")
    else:
        assert r.entropy is None
    if k:
        np.testing.assert_array_equal(r.top_tokens.cpu().numpy(), np.stack([w["top_tokens"] for w in want]))
        _near(r.top_logprobs.cpu(), np.stack([w["top_logprobs"] for w in want]), 3e-5, 2.0 ** -22, "top_logprobs")
    else:
        assert r.top_tokens is None and r.top_logprobs is None
    return r


def _logits(rows, vocab, dtype, seed, scale=3.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = (torch.randn(rows, vocab, generator=g, device="cuda") * scale).to(DTYPES[dtype])
    return x, torch.randint(0, vocab, (rows,), generator=g, device="cuda")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (3, 2, 2), (2, 7, 3), (5, 31, 0), (1, 1000, 20), (7, 1003, 128), (2, 128, 128),
                                          (3, 4096, 1), (2, 16385, 64), (1, 50001, 5), (40, 5003, 8), (700, 257, 4)])
def test_sizes(dtype, rows, vocab, k):
    x, tokens = _logits(rows, vocab, dtype, rows * 1000 + vocab)
    _check(x, tokens, k, 1.0)
    _check(x, tokens, k, 0.7, entropy=False)


@pytest.mark.parametrize("rows", [1, 4, 33, 150, 311])
def test_rows_cut_into_any_number_of_parts(rows):
    x, tokens = _logits(rows, 40003, "bf16", rows)
    _check(x, tokens, 20, 1.3)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_masked_empty_and_special_rows(dtype):
    vocab = 9001
    x, tokens = _logits(12, vocab, dtype, 5)
    inf, low = float("inf"), torch.finfo(DTYPES[dtype]).min
    keep = torch.rand(12, vocab, device="cuda") < 0.002
    x[0] = x[0].masked_fill(~keep[0], -inf)            # fewer allowed tokens than alternatives
    x[1] = -inf                                        # none
    x[2] = low                                         # the type's lowest value everywhere
    x[3] = x[3].masked_fill(~keep[3], low)             # ... as a mask
    x[4] = low
    x[4, 5000:] = -inf
    x[5, 17] = float("nan")
    x[6, 18] = inf
    x[7] = -inf
    x[7, vocab - 1] = 1.0                              # one token left
    tokens[7] = vocab - 1
    tokens[8] = -100
    tokens[9] = vocab
    x[10] = 0.0                                        # all equal
    x[11] = 0.0
    x[11, ::2] = -0.0
    r = profk.logprobs(x, tokens, k=20)
    host, tok = x.float().cpu().numpy(), tokens.cpu().numpy()
    want = [oracle.logprobs_row(host[i], int(tok[i]), 20) for i in range(12)]
    # entries at the lowest value lie further below the maximum than fp32 holds: -inf there
    limit = np.float64(np.finfo(np.float32).max)
    for i in range(12):
        for key, got in (("lse", r.lse), ("logprob", r.logprob), ("entropy", r.entropy), ("top_logprobs", r.top_logprobs)):
            g, w = np.atleast_1d(got[i].cpu().numpy()), np.atleast_1d(np.asarray(want[i][key], dtype=np.float64))
            w = np.where(w < -limit, -np.inf, w)
            if np.isfinite(host[i][~np.isneginf(host[i])]).all() or key != "top_logprobs":
                _near(g, w, 1e-4, 2.0 ** -20, f"{key} of row {i}")
        np.testing.assert_array_equal(r.top_tokens[i].cpu().numpy(), want[i]["top_tokens"], err_msg=f"row {i}")


@pytest.mark.parametrize("order", ["ascending", "descending", "constant", "two values", "late masses"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_orders_that_refill_the_candidate_list(order, dtype):
    vocab = 70001
    ramp = torch.linspace(-8, 8, vocab, device="cuda")
    x = {"ascending": ramp, "descending": ramp.flip(0), "constant": torch.full_like(ramp, 1.5),
         "two values": torch.where(torch.arange(vocab, device="cuda") % 3 == 0, 2.0, 1.0),
         "late masses": torch.where(torch.arange(vocab, device="cuda") > 60000, 5.0, -5.0)}[order]
    for rows in (1, 600):
        many = x.to(DTYPES[dtype]).repeat(rows, 1)
        for k in (1, 20, 128):
            r = profk.logprobs(many, k=k)
            want = oracle.logprobs_row(many[0].float().cpu().numpy(), None, k)
            assert (r.top_tokens == torch.from_numpy(want["top_tokens"]).cuda()).all()
            _near(r.lse.cpu(), np.full(rows, want["lse"]), 3e-5, 2.0 ** -22, "lse")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,masked", [(1, "none"), (2, "front"), (3, "middle"), (300, "none")])
def test_long_rows_and_masked_stretches(dtype, rows, masked):
    """Many batches per part (the bound is renewed on the way), and whole parts of a row without any token."""
    vocab = 1_500_007 if rows < 100 else 200_003
    x, _ = _logits(rows, vocab, dtype, rows)
    if masked == "front":
        x[:, :vocab // 2] = -float("inf")
    elif masked == "middle":
        x[:, vocab // 5:vocab - 100] = -float("inf")
    for k in (3, 30, 100):
        r = profk.logprobs(x, k=k)
        for i in {0, rows - 1}:
            host = x[i].float().cpu().numpy()
            order = np.argsort(-host, kind="stable")[:k]              # (no zeros of either sign are near the largest)
            np.testing.assert_array_equal(r.top_tokens[i].cpu().numpy(), order)
            z = host[np.isfinite(host)].astype(np.float64)
            lse = z.max() + np.log(np.exp(z - z.max()).sum())
            _near(r.lse[i].cpu(), lse, 3e-5, 2.0 ** -22, "lse")
            _near(r.top_logprobs[i].cpu(), host[order] - lse, 3e-5, 2.0 ** -22, "top_logprobs")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,vocab,k,levels", [(2, 131072, 128, 0), (300, 131075, 128, 0), (300, 40001, 100, 0), (2, 200001, 17, 0), (300, 60001, 128, 500), (2, 60001, 64, 40)])
def test_many_alternatives_of_long_rows(dtype, rows, vocab, k, levels):
    """More noted vectors than are read at a time; with `levels`, values that many elements share (lowest index first)."""
    x, _ = _logits(rows, vocab, dtype, vocab + k)
    if levels:
        x = (torch.round(x.float() * (levels / 30)) * (30 / levels) + 0.0).to(x.dtype)
    x[0, 100:vocab - 100] = -float("inf")
    r = profk.logprobs(x, k=k)
    torch.cuda.synchronize()
    for i in sorted({0, 1, rows // 2, rows - 1}):
        host = x[i].double().cpu().numpy()
        order = np.argsort(-host, kind="stable")[:k]
        np.testing.assert_array_equal(r.top_tokens[i].cpu().numpy(), order)
        lse = host.max() + np.log(np.exp(host - host.max()).sum())
        _near(r.top_logprobs[i].cpu(), host[order] - lse, 3e-5, 2.0 ** -22, "top_logprobs")


def test_strides_offsets_and_leading_dimensions():
    base = torch.randn(6, 2100, device="cuda").to(torch.bfloat16)
    for off, vocab in ((0, 2000), (1, 2003), (3, 777), (7, 2093)):
        x = base[:, off:off + vocab]
        _check(x, torch.arange(6, device="cuda"), 9, 1.0)
    x = torch.randn(2, 3, 515, device="cuda")
    r = profk.logprobs(x, torch.zeros(2, 3, dtype=torch.int64, device="cuda"), k=2)
    assert r.lse.shape == r.logprob.shape == r.entropy.shape == (2, 3) and r.top_tokens.shape == (2, 3, 2)
    flat = profk.logprobs(x.view(6, 515), k=2)
    assert torch.equal(flat.lse.view(2, 3), r.lse) and flat.logprob is None
    one = profk.logprobs(x[0, 0])
    assert one.lse.shape == () and torch.equal(one.lse, r.lse[0, 0])


def test_the_same_call_gives_the_same_bits_on_any_stream():
    x, tokens = _logits(37, 60013, "bf16", 9)
    a = profk.logprobs(x, tokens, k=50)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = x.clone()
        b = profk.logprobs(y, tokens, k=50)
    torch.cuda.current_stream().wait_stream(side)
    for p, q in zip(a, b):
        assert torch.equal(p, q)


def test_in_a_graph():
    x, tokens = _logits(8, 30000, "f16", 3)
    want = profk.logprobs(x, tokens, k=8)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = profk.logprobs(x, tokens, k=8)
    graph.replay()
    torch.cuda.synchronize()
    for p, q in zip(got, want):
        assert torch.equal(p, q)


# --- gradient -------------------------------------------------------------------------------------------------------

def _gradient_case(rows, vocab, dtype, k, seed):
    x, tokens = _logits(rows, vocab, dtype, seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1)
    up = [torch.randn(rows, generator=g, device="cuda") for _ in range(3)]
    g_top = torch.randn(rows, k, generator=g, device="cuda") if k else None
    return x, tokens, up, g_top


def _check_gradient(x, tokens, up, g_top, temperature, k, dtype):
    r = profk.logprobs(x, tokens, k=k, temperature=temperature)
    grad = profk.logprobs_backward(x, r.lse, tokens, up[0], entropy=r.entropy, grad_entropy=up[1], grad_lse=up[2],
                                   top_tokens=r.top_tokens, grad_top=g_top, lse_rest=r.lse_rest, temperature=temperature)
    assert grad.dtype == x.dtype and grad.shape == x.shape
    host, got = x.float().cpu().numpy(), grad.float().cpu().numpy().astype(np.float64)
    ulp, least = STEP[dtype]
    for i in range(host.shape[0]):
        top = r.top_tokens[i].cpu().numpy() if k else []
        gt = g_top[i].cpu().numpy().astype(np.float64) if k else []
        want, size = oracle.logprobs_gradient_row(host[i], temperature, int(tokens[i]), float(up[0][i]), float(up[1][i]), float(up[2][i]), top, gt)
        # lse and entropy come from the forward call with its own errors (3e-5, 1e-4 at worst): they move ln p and the factor
        a = np.exp(np.where(np.isneginf(host[i]), -np.inf, host[i].astype(np.float64) / temperature - oracle.logprobs_row(host[i], temperature=temperature)["lse"])) \
            if not np.isneginf(host[i]).all() else 0.0
        moved = a * (abs(float(up[0][i])) + np.sum(np.abs(gt)) + abs(float(up[2][i])) + 50 * abs(float(up[1][i]))) * 3e-5 / temperature
        assert (np.abs(got[i] - want) <= 0.5 * ulp * np.abs(want) + least + 4 * size + moved).all(), f"row {i}"
    return grad


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (2, 7, 3), (3, 1000, 0), (2, 16384, 5), (5, 16387, 128), (2, 40001, 20)])
def test_gradient_sizes(dtype, rows, vocab, k):
    x, tokens, up, g_top = _gradient_case(rows, vocab, dtype, k, vocab + rows)
    _check_gradient(x, tokens, up, g_top, 0.7, k, dtype)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_gradient_of_masked_and_empty_rows(dtype):
    x, tokens, up, g_top = _gradient_case(6, 3001, dtype, 4, 8)
    keep = torch.rand(6, 3001, device="cuda") < 0.01
    x[0] = x[0].masked_fill(~keep[0], -float("inf"))
    x[1] = -float("inf")
    x[2] = torch.finfo(x.dtype).min
    tokens[3] = -1
    tokens[4] = 3001
    grad = _check_gradient(x, tokens, up, g_top, 1.0, 4, dtype)
    assert (grad[1] == 0).all()


def test_gradient_where_token_and_alternatives_coincide():
    x, tokens, up, g_top = _gradient_case(4, 999, "f32", 6, 2)
    tokens = profk.logprobs(x, k=1).top_tokens[:, 0].contiguous()
    _check_gradient(x, tokens, up, g_top, 1.0, 6, "f32")


def test_gradient_of_strided_logits():
    base = torch.randn(5, 1100, device="cuda").to(torch.bfloat16)
    x = base[:, 3:1000]
    up = [torch.randn(5, device="cuda") for _ in range(3)]
    _check_gradient(x, torch.arange(5, device="cuda"), up, None, 1.0, 0, "bf16")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("offset", [1, 2, 3, 5, 7])
def test_gradient_of_logits_at_another_alignment(dtype, offset):
    """Every offset of the logits within 16 bytes against the same values in rows of their own: the same bits."""
    for vocab, pad in ((5003, 9), (4096, 8), (2049, 11)):
        base = torch.randn(7, vocab + pad, device="cuda").to(DTYPES[dtype])
        x = base[:, offset:offset + vocab]
        tokens = torch.arange(7, device="cuda")
        r = profk.logprobs(x, tokens, k=3)
        g = torch.randn(7, device="cuda")
        args = dict(entropy=r.entropy, grad_entropy=g, top_tokens=r.top_tokens, grad_top=torch.randn(7, 3, device="cuda"))
        got = profk.logprobs_backward(x, r.lse, tokens, g, **args)
        assert torch.equal(got, profk.logprobs_backward(x.contiguous(), r.lse, tokens, g, **args))


def test_gradient_against_differences():
    rows, vocab, k, t = 3, 41, 5, 0.8
    x, tokens, up, g_top = _gradient_case(rows, vocab, "f32", k, 21)
    r = profk.logprobs(x, tokens, k=k, temperature=t)
    grad = profk.logprobs_backward(x, r.lse, tokens, up[0], entropy=r.entropy, grad_entropy=up[1], grad_lse=up[2],
                                   top_tokens=r.top_tokens, grad_top=g_top, temperature=t).cpu().numpy()
    host, h = x.cpu().numpy().astype(np.float64), 1e-5
    for i in range(rows):
        rest = (t, int(tokens[i]), float(up[0][i]), float(up[1][i]), float(up[2][i]), r.top_tokens[i].cpu().numpy(), g_top[i].cpu().numpy().astype(np.float64))
        for v in range(vocab):
            a, b = host[i].copy(), host[i].copy()
            a[v] += h
            b[v] -= h
            diff = (oracle.logprobs_loss(a, *rest) - oracle.logprobs_loss(b, *rest)) / (2 * h)
            assert abs(diff - grad[i, v]) <= 1e-4       # h^2 times the third derivative (< 100), and fp32 in the kernel


def test_autograd():
    x, tokens, up, g_top = _gradient_case(4, 2003, "f32", 3, 4)
    leaf = x.clone().requires_grad_(True)
    r = profk.logprobs(leaf, tokens, k=3, temperature=1.5)
    loss = (r.logprob * up[0]).sum() + (r.entropy * up[1]).sum() + (r.lse * up[2]).sum() + (r.top_logprobs * g_top).sum()
    loss.backward()
    want = profk.logprobs_backward(x, r.lse.detach(), tokens, up[0], entropy=r.entropy.detach(), grad_entropy=up[1], grad_lse=up[2],
                                   top_tokens=r.top_tokens, grad_top=g_top, lse_rest=r.lse_rest, temperature=1.5)
    assert torch.equal(leaf.grad, want)
    leaf.grad = None
    profk.logprobs(leaf, tokens, entropy=False).logprob.sum().backward()      # parts that no loss uses bring no gradient
    ref = torch.log_softmax(x.double(), -1)
    p = ref.exp()
    want = -p
    want[torch.arange(4), tokens] += 1
    assert (leaf.grad.double() - want).abs().max() < 1e-5


# --- refusals -------------------------------------------------------------------------------------------------------

def test_refusals():
    x = torch.randn(4, 100, device="cuda")
    tok = torch.zeros(4, dtype=torch.int64, device="cuda")
    lse = torch.zeros(4, device="cuda")
    bad = [lambda: profk.logprobs(x, k=101), lambda: profk.logprobs(torch.randn(4, 200, device="cuda"), k=129), lambda: profk.logprobs(x, k=-1),
           lambda: profk.logprobs(x, temperature=0.0), lambda: profk.logprobs(x, temperature=-1.0), lambda: profk.logprobs(x, temperature=float("nan")),
           lambda: profk.logprobs(x, temperature=float("inf")), lambda: profk.logprobs(x.double()), lambda: profk.logprobs(x.cpu()),
           lambda: profk.logprobs(x.t()), lambda: profk.logprobs(x[:0]), lambda: profk.logprobs(x, tok.int()), lambda: profk.logprobs(x, tok[:3]),
           lambda: profk.logprobs(x, tok.cpu()), lambda: profk.logprobs(x.expand(2, 4, 100)[:, 0:1].expand(2, 4, 100)),
           lambda: profk.logprobs_backward(x, lse.double(), tok, lse), lambda: profk.logprobs_backward(x, lse, None, lse),
           lambda: profk.logprobs_backward(x, lse, tok, grad_entropy=lse), lambda: profk.logprobs_backward(x, lse, grad_top=torch.zeros(4, 2, device="cuda"))]
    for n, call in enumerate(bad):
        with pytest.raises(profk.ProfkError):
            call()
            pytest.fail(f"call {n} was not refused")
    _check(x, tok, 3, 1.0)
