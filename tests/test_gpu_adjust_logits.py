"""Penalties, biases and masks over logits, against the oracle on a GPU.

Tolerances.  Each step is one fp32 operation, off by 2^-24 of its result; the oracle returns the sum of those magnitudes.  The
result is rounded once to its type.  Logits that nothing applies to keep their bits."""
import numpy as np
import pytest
import torch

import paper_2608_12573_b200 as profk
from oracle import prompt as oracle
from paper_2608_12573_b200 import _build

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    _build.build()
    profk.lib()
    torch.cuda.set_device(0)


def _gen(seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _logits(rows, vocab, dtype="f32", seed=0):
    return (torch.randn(rows, vocab, generator=_gen(seed), device="cuda") * 4).to(DTYPES[dtype])


def _mask(rows, vocab, share=0.5, seed=0):
    rng = np.random.default_rng(seed)
    bits = rng.random((rows, -(-vocab // 32), 32)) < share
    words = (bits.astype(np.uint32) << np.arange(32, dtype=np.uint32)).sum(-1, dtype=np.uint32)
    return torch.from_numpy(words.view(np.int32)).cuda()


def _bits(t):
    return t.view(torch.int32 if t.dtype == torch.float32 else torch.int16)


def _check(x, tokens=None, lengths=None, prompts=None, out=None, result=None, **how):
    """x (rows, V)."""
    before = x.clone()
    got = profk.adjust_logits(x, tokens, lengths, prompts, out=out, **how) if result is None else result
    torch.cuda.synchronize()
    assert got.shape == x.shape and got.dtype == x.dtype
    rows = x.shape[0]

    def row(name, r, default):
        v = how.get(name, default)
        return float(v[r]) if isinstance(v, torch.Tensor) else v

    def line(t, r):
        return None if t is None else (t if t.dim() == 1 else t[r]).cpu().numpy()

    host, values = before.double().cpu().numpy(), got.double().cpu().numpy()
    eps = torch.finfo(x.dtype).eps / 2
    for r in range(rows):
        history = [] if tokens is None else line(tokens, r)
        if lengths is not None:
            history = history[:max(0, int(lengths[r]))]
        bt, bv = line(how.get("bias_tokens"), r), line(how.get("bias_values"), r)
        want, size, changed = oracle.adjust_row(host[r], history, 0 if prompts is None else int(prompts[r]), row("repetition", r, 1.0), row("frequency", r, 0.0),
                                                row("presence", r, 0.0), () if bt is None else bt, () if bv is None else bv, line(how.get("mask"), r))
        same = torch.from_numpy(~changed).cuda()
        assert torch.equal(_bits(got[r])[same], _bits(before[r])[same]), f"row {r}: logits that nothing applies to changed"
        # (what lies beyond the type's largest value by half a step or more rounds to infinity)
        want = np.where(np.abs(want) >= torch.finfo(x.dtype).max * (1 + eps / 2), np.copysign(np.inf, want), want)
        off = ~np.isfinite(want)
        assert np.array_equal(values[r][off], want[off], equal_nan=True), f"row {r}"
        allowed = size * 2.0 ** -23 + eps * np.abs(np.where(off, 0, want)) + torch.finfo(x.dtype).tiny
        wrong = np.abs(np.where(off, 0, values[r]) - np.where(off, 0, want)) > allowed
        assert not wrong.any(), f"row {r}: {values[r][wrong][:4]} for {want[wrong][:4]} at {wrong.nonzero()[0][:4]}"
    return got


def _history(rows, vocab, n, seed=1):
    g = _gen(seed)
    tokens = torch.randint(0, vocab, (rows, n), generator=g, device="cuda")
    tokens[:, ::3] = tokens[:, :1].clone()                       # one token again and again
    return tokens


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("vocab", [1, 7, 8, 31, 33, 1000, 4099, 131071])
@pytest.mark.parametrize("history", [0, 1, 37, 5000])
def test_sizes(dtype, vocab, history):
    rows = 3
    x = _logits(rows, vocab, dtype)
    how = dict(repetition=1.3, frequency=0.25, presence=0.5, mask=_mask(rows, vocab))
    tokens = _history(rows, vocab, history) if history else None
    lengths = torch.tensor([history, history // 2, 0], dtype=torch.int32, device="cuda") if history else None
    prompts = torch.tensor([history // 3, history, 0], dtype=torch.int32, device="cuda") if history else None
    want = _check(x, tokens, lengths, prompts, **how)
    place = x.clone()
    assert profk.adjust_logits(place, tokens, lengths, prompts, out=place, **how) is place and torch.equal(_bits(place), _bits(want))


def test_vocabularies_beyond_one_round_of_counters():
    x = _logits(2, 600001, "bf16")
    tokens = _history(2, 600001, 3000)
    bias_tokens = torch.tensor([[0, 262143, 262144, 600000, 300000], [599999, 524288, 5, 5, 1]], device="cuda")
    _check(x, tokens, repetition=2.0, frequency=0.5, bias_tokens=bias_tokens, bias_values=torch.randn(2, 5, generator=_gen(), device="cuda"), mask=_mask(2, 600001, 0.9))


def test_rows_at_any_alignment():
    for shift in range(9):
        wide, target = torch.zeros(4, 1100, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, 1203, dtype=torch.bfloat16, device="cuda")
        x = wide[:, shift:shift + 1000]
        x.copy_(_logits(4, 1000, "bf16"))
        for out in (None, target[:, 3:1003]):
            _check(x, _history(4, 1000, 50), out=out, repetition=1.5, bias_tokens=torch.tensor([0, 999, 17], device="cuda"),
                   bias_values=torch.tensor([1.0, 2.0, -3.0], device="cuda"), mask=_mask(4, 1000, 0.8))
        assert (target[:, :3] == 0).all() and (target[:, 1003:] == 0).all()
        _check(x, mask=_mask(4, 1000, 0.8)[0])


def test_values_per_row():
    rows, vocab = 5, 2000
    g = _gen(4)
    each = lambda: torch.rand(rows, generator=g, device="cuda") + 0.5  # noqa: E731
    _check(_logits(rows, vocab), _history(rows, vocab, 300), repetition=each(), frequency=-each(), presence=each())
    _check(_logits(rows, vocab), _history(1, vocab, 300)[0], repetition=each())          # one history for all


def test_tokens_outside_the_vocabulary_are_passed_over():
    x = _logits(2, 100)
    tokens = torch.tensor([[-1, 100, 5, -100, 2 ** 40, 5, -(2 ** 62), 99], [-5] * 8], device="cuda")
    for offset in range(4):
        base = torch.zeros(2, 104, device="cuda")
        y = base[:, offset:offset + 100]
        y.copy_(x)
        _check(y, tokens, frequency=1.0, presence=2.0, bias_tokens=tokens, bias_values=torch.ones(2, 8, device="cuda"), out=y.clone())
        assert torch.equal(y, x)


def test_lengths_and_prompts_outside_the_history():
    x, tokens = _logits(4, 50), _history(4, 50, 20)
    lengths = torch.tensor([-3, 1 << 30, 20, 10], dtype=torch.int32, device="cuda")
    prompts = torch.tensor([5, -5, 1 << 30, 10], dtype=torch.int32, device="cuda")
    _check(x, tokens, lengths, prompts, repetition=0.5, frequency=0.1, presence=0.2)


@pytest.mark.parametrize("n", [1, 300, 8192])
def test_biases_named_more_than_once(n):
    x = _logits(3, 500, "f32")
    g = _gen(5)
    at, values = torch.randint(0, 500, (3, n), generator=g, device="cuda"), torch.randn(3, n, generator=g, device="cuda")
    got = _check(x, bias_tokens=at, bias_values=values)
    for _ in range(3):
        assert torch.equal(profk.adjust_logits(x, bias_tokens=at, bias_values=values), got)


def test_special_values():
    x = _logits(2, 64)
    x[:, 0], x[:, 1], x[:, 2], x[:, 3] = float("nan"), float("inf"), -float("inf"), 0.0
    x[:, 4] = -0.0
    x[:, 5] = torch.finfo(torch.float32).min
    x.view(torch.int32)[:, 6] = 0x7FA12345               # a NaN with a payload, that nothing applies to
    tokens = torch.tensor([[0, 1, 2, 3, 4, 5]] * 2, device="cuda")
    mask = torch.full((2, 2), -1, dtype=torch.int32, device="cuda")
    mask[1] = 0                                          # nothing is allowed
    got = _check(x, tokens, repetition=2.0, mask=mask, prompts=torch.tensor([3, 0], dtype=torch.int32, device="cuda"))
    assert torch.isneginf(got[1]).all()
    # biases of infinity ban and force; the mask wins
    values = torch.tensor([float("inf"), -float("inf"), 1.0], device="cuda")
    got = _check(_logits(2, 64), bias_tokens=torch.tensor([7, 8, 40], device="cuda"), bias_values=values, mask=mask)
    assert torch.isposinf(got[0, 7]) and torch.isneginf(got[0, 8])


def test_shapes():
    x, tokens = _logits(6, 300), _history(6, 300, 40)
    want = profk.adjust_logits(x, tokens, repetition=1.2, mask=_mask(6, 300))
    got = profk.adjust_logits(x.view(2, 3, 300), tokens.view(2, 3, 40), repetition=1.2, mask=_mask(6, 300).view(2, 3, 10))
    assert torch.equal(got.view(6, 300), want)
    assert torch.equal(profk.adjust_logits(x[4], tokens[4], repetition=1.2, mask=_mask(6, 300)[4]), want[4])
    assert torch.equal(profk.adjust_logits(x[::2], tokens[::2], repetition=1.2, mask=_mask(6, 300)[::2]), want[::2])
    assert profk.adjust_logits(x[:0], tokens[:0]).shape == (0, 300)
    assert torch.equal(profk.adjust_logits(x), x)
    assert torch.equal(profk.adjust_logits(x, tokens[:, :0]), x)


def test_many_rows_and_long_histories():
    x = _logits(300, 5000, "f16")
    _check(x, _history(300, 5000, 700), frequency=0.01, repetition=1.1)
    x = _logits(1, 40000, "f32")
    _check(x, _history(1, 40000, 100000), frequency=0.001, presence=0.1, prompts=torch.tensor([50000], dtype=torch.int32, device="cuda"))


def test_streams_and_graphs():
    x, tokens, mask = _logits(4, 1000), _history(4, 1000, 60), _mask(4, 1000)
    want = profk.adjust_logits(x, tokens, repetition=1.5, mask=mask)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = profk.adjust_logits(x, tokens, repetition=1.5, mask=mask)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    torch.cuda.synchronize()
    graph, y = torch.cuda.CUDAGraph(), x.clone()
    with torch.cuda.graph(graph):
        profk.adjust_logits(y, tokens, repetition=1.5, mask=mask, out=y)
    y.copy_(x)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)


def test_refusals():
    x, tokens = _logits(3, 64), _history(3, 64, 10)
    n = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    at, values = torch.zeros(3, 2, dtype=torch.int64, device="cuda"), torch.zeros(3, 2, device="cuda")
    call = profk.adjust_logits
    bad = [lambda: call(x.double()), lambda: call(x.cpu()), lambda: call(x, tokens.int()), lambda: call(x, tokens[:2]), lambda: call(x, tokens, n.long()), lambda: call(x, tokens, n[:2]),
           lambda: call(x, None, n), lambda: call(x, None, None, n), lambda: call(x, tokens, repetition=0.0), lambda: call(x, tokens, repetition=-1.0),
           lambda: call(x, tokens, repetition=float("nan")), lambda: call(x, tokens, frequency=float("inf")), lambda: call(x, tokens, presence=1e39),
           lambda: call(x, tokens, repetition=torch.ones(2, device="cuda")), lambda: call(x, tokens, repetition=torch.ones(3, device="cuda").double()),
           lambda: call(x, bias_tokens=at), lambda: call(x, bias_values=values), lambda: call(x, bias_tokens=at, bias_values=values[:, :1]),
           lambda: call(x, bias_tokens=at.int(), bias_values=values), lambda: call(x, bias_tokens=at.new_zeros(8193), bias_values=values.new_zeros(8193)),
           lambda: call(x, mask=_mask(3, 65)), lambda: call(x, mask=_mask(2, 64)), lambda: call(x, mask=_mask(3, 64).long()), lambda: call(x, out=x.half()),
           lambda: call(x, out=x[:2]), lambda: call(x, out=x.t().contiguous().t()), lambda: call(x.t()), lambda: call(x.clone().requires_grad_(True)),
           lambda: call(x, bias_tokens=at, bias_values=values.clone().requires_grad_(True)), lambda: call(x, "tokens"), lambda: call(x, tokens.cpu())]
    wide = torch.zeros(3, 130, device="cuda")
    bad += [lambda: call(wide[:, :64], out=wide[:, 32:96]), lambda: call(wide[:, :64], out=wide[:, 64:128])]
    for i, f in enumerate(bad):
        with pytest.raises(profk.ProfkError):
            f()
            pytest.fail(f"call {i} was not refused")
    assert torch.equal(call(x), x)
