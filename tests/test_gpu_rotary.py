"""Rotary positions, and appending to a paged cache with them, against the oracle on a GPU.

Tolerances.  An angle is off by 2^-33 turns (32 bits of it are kept: 2^-30 radians), 2^-24 of what lies beyond the nearest
quarter turn (pi / 4 at most) and, through the 53 bits of the frequency in turns, 3 * 2^-54 of itself; cosine and sine add 2 units in the
last place, the magnitude one: 5 * 2^-24 in all.  The two products and their sum add 2^-24 each.  So an element is off by the
sum of its pair's magnitudes times 2^-21 + |angle| 2^-52, and half a unit in the last place of its type."""
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


def _randn(*shape, dtype="bf16", seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(DTYPES[dtype])


def _host(t):
    return t.detach().double().cpu().numpy()


def _near(got, x, positions, frequencies, **how):
    """got, x (tokens, heads, dim)."""
    want, size, angle = oracle.rotary(_host(x), positions.cpu().numpy(), _host(frequencies), **how)
    allowed = size * (2.0 ** -21 + angle * 2.0 ** -52) + torch.finfo(got.dtype).eps / 2 * np.abs(want) + torch.finfo(got.dtype).tiny
    off = np.abs(_host(got) - want)
    assert (off <= allowed).all(), f"{off.max()} at {np.unravel_index((off - allowed).argmax(), off.shape)}"


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,dim,turned", [(1, 1, 2, 2), (3, 5, 64, 64), (7, 1, 128, 32), (300, 3, 80, 20), (2, 2, 96, 6), (1000, 8, 128, 128), (5, 2, 1024, 1024),
                                                     (9, 33, 24, 16), (4000, 2, 256, 64), (3, 2, 7, 6)])
def test_sizes(dtype, interleaved, tokens, heads, dim, turned):
    x, f = _randn(tokens, heads, dim, dtype=dtype), profk.rotary_frequencies(turned)
    at = torch.arange(tokens, device="cuda") * 37
    got = profk.rotary(x, at, f, interleaved=interleaved, magnitude=1.25)
    _near(got, x, at, f, interleaved=interleaved, magnitude=1.25)
    assert torch.equal(got[..., turned:], x[..., turned:])


@pytest.mark.parametrize("at", [0, -1, 131071, 10 ** 6 + 3, -(10 ** 7), 2 ** 31 - 1, 2 ** 40 + 12345])
def test_far_positions(at):
    x, f = _randn(4, 2, 64, dtype="f32"), profk.rotary_frequencies(64)
    positions = torch.tensor([at, at + 1, at - 1, at], device="cuda")
    for inverse in (False, True):
        _near(profk.rotary(x, positions, f, inverse=inverse), x, positions, f, inverse=inverse)
    if at == 0:
        assert torch.equal(profk.rotary(x, positions, f)[0], x[0])


def test_frequencies_of_any_kind():
    x = _randn(6, 2, 12, dtype="f32")
    f = torch.tensor([0.0, -0.3, 7.0, 1e-12, np.pi, 1e5], dtype=torch.float64, device="cuda")
    positions = torch.arange(6, device="cuda") * 1001
    _near(profk.rotary(x, positions, f), x, positions, f)


def test_frequencies_for_longer_contexts():
    plain = profk.rotary_frequencies(64, device="cpu")
    i = torch.arange(32, dtype=torch.float64)
    assert torch.allclose(plain, 10000.0 ** (-i / 32), rtol=1e-14, atol=0)
    assert torch.allclose(profk.rotary_frequencies(64, stretch=4.0, device="cpu"), plain / 4, rtol=1e-15, atol=0)
    mixed = profk.rotary_frequencies(64, stretch=4.0, context=4096, keep=32, slow=1, device="cpu")
    turns = plain * 4096 / (2 * np.pi)
    assert torch.equal(mixed[turns >= 32], plain[turns >= 32]) and torch.equal(mixed[turns <= 1], plain[turns <= 1] / 4)
    between = (turns < 32) & (turns > 1)
    assert between.any() and (mixed[between] < plain[between]).all() and (mixed[between] > plain[between] / 4).all()
    for bad in (dict(dim=7), dict(dim=0), dict(dim=8, base=0.0), dict(dim=8, stretch=0.0), dict(dim=8, context=0), dict(dim=8, context=9, keep=1.0, slow=1.0)):
        with pytest.raises(profk.ProfkError):
            profk.rotary_frequencies(device="cpu", **bad)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_strides_and_alignments_do_not_matter(dtype, interleaved):
    x, f = _randn(2, 15, 6, 64, dtype=dtype), profk.rotary_frequencies(48)
    at = torch.arange(15, device="cuda").expand(2, 15)
    want = profk.rotary(x, at, f, interleaved=interleaved)
    _near(want.flatten(0, 1), x.flatten(0, 1), at.reshape(-1), f, interleaved=interleaved)
    for shift in (0, 1, 8):
        wide = torch.zeros(2, 15, 9, 64 + 16, dtype=x.dtype, device="cuda")
        view = wide[:, :, 2:8, shift:shift + 64]
        view.copy_(x)
        assert torch.equal(profk.rotary(view, at, f, interleaved=interleaved), want)
    by_head = x.transpose(1, 2).contiguous().transpose(1, 2)
    assert torch.equal(profk.rotary(by_head, at, f, interleaved=interleaved), want)
    assert torch.equal(profk.rotary(x.transpose(0, 1), at.t(), f, interleaved=interleaved), want.transpose(0, 1))
    assert torch.equal(profk.rotary(x, torch.arange(15, device="cuda"), f, interleaved=interleaved), want)
    one = x[:, :, :1].expand(2, 15, 6, 64)
    assert torch.equal(profk.rotary(one, at, f, interleaved=interleaved), want[:, :, :1].expand(2, 15, 6, 64))
    assert torch.equal(profk.rotary(x[0, 3], at[0, 3], f, interleaved=interleaved), want[0, 3])


def test_a_head_s_other_elements_keep_their_bits_and_pairs_their_own_faults():
    x, f = _randn(3, 2, 64, dtype="f32"), profk.rotary_frequencies(32)
    x.view(torch.int32)[1, 0, 40] = 0x7FA12345           # a NaN with a payload, where nothing is turned
    x[2, 1, 3] = float("inf")                            # meets element 19 only
    at = torch.arange(3, device="cuda")
    got = profk.rotary(x, at, f)
    assert torch.equal(got.view(torch.int32)[..., 32:], x.view(torch.int32)[..., 32:])
    bad = ~torch.isfinite(got[2, 1])
    assert bad.nonzero().flatten().tolist() == [3, 19]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("interleaved", [False, True])
def test_wide_heads_of_many_tokens(dtype, interleaved):
    """As many pairs and tokens as a CTA's room for angles is shortest for."""
    x, f = _randn(9001, 1, 1024, dtype=dtype), profk.rotary_frequencies(1024)
    at = torch.arange(9001, device="cuda") % 700
    got = profk.rotary(x, at, f, interleaved=interleaved)
    rows = torch.cat([torch.arange(40, device="cuda"), torch.arange(8970, 9001, device="cuda")])
    _near(got[rows], x[rows], at[rows], f, interleaved=interleaved)
    assert torch.equal(got[700:1400], profk.rotary(x[700:1400], at[:700], f, interleaved=interleaved))


def test_no_tokens():
    f = profk.rotary_frequencies(8)
    assert profk.rotary(_randn(0, 4, 8), torch.zeros(0, dtype=torch.int64, device="cuda"), f).shape == (0, 4, 8)
    assert profk.rotary(_randn(2, 0, 4, 8), torch.zeros(2, 0, dtype=torch.int64, device="cuda"), f).shape == (2, 0, 4, 8)


# --- gradient -------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient(dtype, interleaved):
    x, g, f = _randn(50, 3, 96, dtype=dtype).requires_grad_(True), _randn(50, 3, 96, dtype=dtype, seed=1), profk.rotary_frequencies(64)
    at = torch.arange(50, device="cuda") * 11
    y = profk.rotary(x, at, f, interleaved=interleaved, magnitude=0.8)
    grad, = torch.autograd.grad(y, x, g)
    _near(grad, g, at, f, interleaved=interleaved, magnitude=0.8, inverse=True)


def test_gradient_against_differences():
    x, f = _randn(4, 2, 8, dtype="f32").requires_grad_(True), profk.rotary_frequencies(6)
    at, w = torch.tensor([0, 1, 5, 900], device="cuda"), _randn(4, 2, 8, dtype="f32", seed=2)
    grad, = torch.autograd.grad((profk.rotary(x, at, f, magnitude=1.1) * w).sum(), x)
    for seed in range(4):
        d = _randn(4, 2, 8, dtype="f32", seed=10 + seed)
        with torch.no_grad():       # (linear: the difference is exact up to rounding, 2^-21 of sums of 64 products of order 10)
            diff = ((profk.rotary(x + d, at, f, magnitude=1.1) - profk.rotary(x - d, at, f, magnitude=1.1)).double() * w.double()).sum() / 2
        assert abs((grad.double() * d.double()).sum() - diff) < 64 * 10 * 2.0 ** -21


def test_gradients_of_broadcasts_and_second_derivatives():
    f, at = profk.rotary_frequencies(8), torch.arange(5, device="cuda")
    x = _randn(5, 1, 8, dtype="f32").requires_grad_(True)
    y = profk.rotary(x.expand(5, 7, 8), at, f)
    y.sum().backward()                                   # (an upstream gradient of strides zero)
    ones = torch.ones(5, 1, 8, device="cuda")
    assert torch.allclose(x.grad, 7 * profk.rotary(ones, at, f, inverse=True), rtol=2.0 ** -20, atol=2.0 ** -19)
    # d/dx of |y|^2 = 2 m^2 x, and of its gradient's square 8 m^4 x
    x = _randn(5, 2, 8, dtype="f32").requires_grad_(True)
    grad, = torch.autograd.grad((profk.rotary(x, at, f, magnitude=2.0) ** 2).sum(), x, create_graph=True)
    assert torch.allclose(grad, 8 * x, rtol=2.0 ** -19, atol=2.0 ** -18)
    second, = torch.autograd.grad((grad ** 2).sum(), x)
    assert torch.allclose(second, 128 * x, rtol=2.0 ** -17, atol=2.0 ** -14)


def test_upstream_gradients_of_any_layout():
    f, at = profk.rotary_frequencies(8), torch.arange(5, device="cuda")
    x = _randn(2, 3, 4, 5, 6, 8, dtype="f32").requires_grad_(True)
    w = _randn(6, 4, 5, 2, 8, 3, dtype="f32", seed=1)
    grad, = torch.autograd.grad((profk.rotary(x, at, f).permute(4, 2, 3, 0, 5, 1) * w).sum(), x)
    assert torch.equal(grad, profk.rotary(w.permute(3, 5, 1, 2, 0, 4).contiguous(), at, f, inverse=True))
    x = _randn(2, 5, 6, 8, dtype="f32").requires_grad_(True)
    w = _randn(8, 2, 6, 5, dtype="f32", seed=1)
    grad, = torch.autograd.grad((profk.rotary(x, at, f).permute(3, 0, 2, 1) * w).sum(), x)
    assert torch.equal(grad, profk.rotary(w.permute(1, 3, 2, 0).contiguous(), at, f, inverse=True))


def test_streams_graphs_and_repeated_calls():
    x, f, at = _randn(100, 4, 64).requires_grad_(True), profk.rotary_frequencies(64), torch.arange(100, device="cuda")
    g = _randn(100, 4, 64, seed=3)
    # (a leaf of its own: torch does not capture a backward pass while an eager graph of the same leaf is alive)
    eager = x.detach().clone().requires_grad_(True)
    want = profk.rotary(eager, at, f)
    want_grad, = torch.autograd.grad(want, eager, g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = profk.rotary(eager, at, f)
        grad, = torch.autograd.grad(got, eager, g)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and torch.equal(grad, want_grad)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = profk.rotary(x, at, f)
        grad, = torch.autograd.grad(got, x, g)
    with torch.no_grad():
        x.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, 2 * want) and torch.equal(grad, want_grad)


def test_refusals():
    x, f, at = _randn(6, 2, 8), profk.rotary_frequencies(8), torch.arange(6, device="cuda")
    import torch.autograd.forward_ad as forward

    bad = [lambda: profk.rotary(x.double(), at, f), lambda: profk.rotary(x.cpu(), at, f), lambda: profk.rotary(x, at.int(), f), lambda: profk.rotary(x, at[:5], f),
           lambda: profk.rotary(x, at.cpu(), f), lambda: profk.rotary(x, at, f.float()), lambda: profk.rotary(x, at, f.cpu()), lambda: profk.rotary(x, at, f[:0]),
           lambda: profk.rotary(x[..., :6], at, f), lambda: profk.rotary(x[..., ::2], at, f[:1]), lambda: profk.rotary(x, at, f, magnitude=float("inf")),
           lambda: profk.rotary(x, at, f, magnitude="2"), lambda: profk.rotary(x[0, 0], at[0], f), lambda: profk.rotary(_randn(1, 2, 1026), at[:1], f),
           lambda: profk.rotary(x, at, f.clone().requires_grad_(True)), lambda: profk.rotary(x, at[:, None].expand(6, 6), f),
           lambda: profk.rotary(_randn(2, 3, 4, 2, 8).permute(2, 1, 0, 3, 4), torch.zeros(2, dtype=torch.int64, device="cuda"), f)]
    for n, call in enumerate(bad):
        with pytest.raises(profk.ProfkError):
            call()
            pytest.fail(f"call {n} was not refused")
    with forward.dual_level(), pytest.raises(RuntimeError):
        profk.rotary(forward.make_dual(x, torch.ones_like(x)), at, f)


# --- appending ------------------------------------------------------------------------------------------------------

def _cache(lengths, kv_heads, dim, page, dtype, tokens_first=False, spare=3, width=None, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    need = [-(-max(n, 0) // page) for n in lengths]
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    tables = torch.full((len(lengths), max(need + [1]) if width is None else width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        n = min(n, tables.shape[1])
        tables[i, :n] = order[at:at + n]
        at += n
    shape = (pages, page, kv_heads, dim) if tokens_first else (pages, kv_heads, page, dim)
    k, v = (torch.randn(shape, generator=g, device="cuda").to(DTYPES[dtype]) for _ in range(2))
    return (k.transpose(1, 2), v.transpose(1, 2), tables) if tokens_first else (k, v, tables)


def _append(k_pages, v_pages, tables, lengths, q, k, v, f, starts=None, positions=None, interleaved=False, magnitude=1.0):
    """Calls it and compares everything with the oracle: turned values as `rotary` has them, bit for bit, in the oracle's places."""
    lengths_t = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    starts_t = None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda")
    want_k, want_v = _host(k_pages), _host(v_pages)
    lead = k.shape[:-2]
    rows = int(np.prod(lead))
    seq, place = oracle.places(lengths, rows, starts)
    at = torch.tensor(place, device="cuda") if positions is None else positions.reshape(-1)
    turned = profk.rotary(k.reshape(rows, *k.shape[-2:]), at, f, interleaved=interleaved, magnitude=magnitude)
    oracle.append(want_k, _host(turned), tables.cpu().numpy(), lengths, starts)
    oracle.append(want_v, _host(v.reshape(rows, *v.shape[-2:])), tables.cpu().numpy(), lengths, starts)
    versions = k_pages._version, v_pages._version
    got = profk.pages_append_rotary(k_pages, v_pages, tables, lengths_t, q, k, v, f, starts=starts_t, positions=positions, interleaved=interleaved, magnitude=magnitude)
    assert np.array_equal(_host(k_pages), want_k, equal_nan=True) and np.array_equal(_host(v_pages), want_v, equal_nan=True)
    if rows:
        assert k_pages._version > versions[0] and v_pages._version > versions[1]
    if q is None:
        assert got is None
        return
    want_q = profk.rotary(q.reshape(rows, *q.shape[-2:]), at, f, interleaved=interleaved, magnitude=magnitude)
    want_q[torch.tensor(seq < 0, device="cuda")] = 0
    assert got.shape == q.shape and torch.equal(got.reshape(want_q.shape), want_q)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("page,tokens_first", [(1, False), (7, True), (16, False), (64, True)])
def test_append_one_token(dtype, interleaved, page, tokens_first):
    lengths = [1, 5, 16, 17, 64, 130]
    cache = _cache(lengths, 2, 64, page, dtype, tokens_first)
    q, k, v = _randn(6, 8, 64, dtype=dtype), _randn(6, 2, 64, dtype=dtype, seed=1), _randn(6, 2, 64, dtype=dtype, seed=2)
    _append(*cache, lengths, q, k, v, profk.rotary_frequencies(32), interleaved=interleaved, magnitude=1.5)


@pytest.mark.parametrize("dim,turned", [(8, 8), (40, 20), (128, 128), (256, 64)])
def test_append_chunks(dim, turned):
    lengths = [40, 33, 100]
    joint = _randn(3, 33, 9, dim)                        # queries, keys and values side by side
    q, k, v = joint[:, :, :5], joint[:, :, 5:7], joint[:, :, 7:]
    _append(*_cache(lengths, 2, dim, 24, "bf16"), lengths, q, k, v, profk.rotary_frequencies(turned))


@pytest.mark.parametrize("starts", [[0, 3, 3, 10, 10, 57], [2, 2, 9, 9, 9, 50], [0, 0, 0, 0, 0, 57], [57, 57, 57, 57, 57, 57], [0, 57, 57, 57, 57, 57]])
def test_append_ragged(starts):
    lengths = [60 if b > a else 9 for a, b in zip(starts, starts[1:])]
    q, k, v = _randn(57, 4, 64, dtype="f16"), _randn(57, 2, 64, dtype="f16", seed=1), _randn(57, 2, 64, dtype="f16", seed=2)
    _append(*_cache(lengths, 2, 64, 16, "f16"), lengths, q, k, v, profk.rotary_frequencies(64), starts=starts)


def test_append_many_ragged_sequences():
    news = [(i * 7) % 5 for i in range(1500)]
    starts = np.concatenate([[0], np.cumsum(news)]).tolist()
    lengths = [n + (i % 9) for i, n in enumerate(news)]
    rows = starts[-1] + 6                                # rows behind the last sequence
    q, k, v = _randn(rows, 2, 16), _randn(rows, 1, 16, seed=1), _randn(rows, 1, 16, seed=2)
    _append(*_cache(lengths, 1, 16, 4, "bf16"), lengths, q, k, v, profk.rotary_frequencies(16), starts=starts)


def test_append_given_positions_and_without_queries():
    lengths = [10, 20]
    cache, f = _cache(lengths, 2, 64, 16, "bf16"), profk.rotary_frequencies(64)
    q, k, v = _randn(2, 6, 3, 64), _randn(2, 6, 2, 64, seed=1), _randn(2, 6, 2, 64, seed=2)
    _append(*cache, lengths, q, k, v, f, positions=torch.randint(-10 ** 6, 10 ** 6, (2, 6), device="cuda"))
    _append(*cache, lengths, None, k, v, f)
    _append(*cache, lengths, q.flatten(0, 1), k.flatten(0, 1), v.flatten(0, 1), f, starts=[0, 5, 12], positions=torch.arange(24, device="cuda")[::2])


def test_tokens_without_a_place_are_turned_only():
    lengths = [3, 70, -2, 40]                            # fewer tokens than are new; past the table; negative; a page that is not there
    k_pages, v_pages, tables = _cache([3, 64, 0, 40], 2, 64, 16, "bf16", width=4)
    tables[3, 1], tables[3, 2] = -1, k_pages.shape[0]
    q, k, v = _randn(4, 9, 3, 64), _randn(4, 9, 2, 64, seed=1), _randn(4, 9, 2, 64, seed=2)
    _append(k_pages, v_pages, tables, lengths, q, k, v, profk.rotary_frequencies(64))


def test_append_nothing():
    k_pages, v_pages, tables = _cache([3, 4], 2, 64, 16, "bf16")
    f = profk.rotary_frequencies(64)
    _append(k_pages, v_pages, tables, [3, 4], _randn(2, 0, 3, 64), _randn(2, 0, 2, 64), _randn(2, 0, 2, 64), f)
    _append(k_pages, v_pages, tables, [3, 4], _randn(0, 3, 64), _randn(0, 2, 64), _randn(0, 2, 64), f, starts=[0, 0, 0])


def test_append_in_a_graph_and_on_a_stream():
    lengths, f = torch.tensor([20, 31], dtype=torch.int32, device="cuda"), profk.rotary_frequencies(64)
    k_pages, v_pages, tables = _cache([40, 40], 2, 64, 16, "bf16")
    q, k, v = _randn(2, 4, 64), _randn(2, 2, 64, seed=1), _randn(2, 2, 64, seed=2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = profk.pages_append_rotary(k_pages, v_pages, tables, lengths, q, k, v, f)
    lengths += 1
    graph.replay()
    torch.cuda.synchronize()
    before = k_pages.clone(), got.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = profk.pages_append_rotary(k_pages, v_pages, tables, lengths, q, k, v, f)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(k_pages, before[0]) and torch.equal(again, before[1])
    assert torch.equal(again, profk.rotary(q, lengths.long() - 1, f))


def test_append_refusals():
    lengths = torch.tensor([10, 20], dtype=torch.int32, device="cuda")
    kp, vp, tables = _cache([10, 20], 2, 64, 16, "bf16")
    q, k, v, f = _randn(2, 4, 64), _randn(2, 2, 64), _randn(2, 2, 64), profk.rotary_frequencies(64)
    starts = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    call = profk.pages_append_rotary
    before = kp.clone()
    bad = [lambda: call(kp, vp, tables, lengths, q.float(), k, v, f), lambda: call(kp, vp, tables, lengths, q, k.half(), v.half(), f), lambda: call(kp, vp[:-1], tables, lengths, q, k, v, f),
           lambda: call(kp, vp, tables.long(), lengths, q, k, v, f), lambda: call(kp, vp, tables, lengths[:1], q, k, v, f), lambda: call(kp, vp, tables, lengths, q[:1], k, v, f),
           lambda: call(kp, vp, tables, lengths, q, k[:, :1], v[:, :1], f), lambda: call(kp, vp, tables, lengths, q, k[..., :32], v[..., :32], f),
           lambda: call(kp, vp, tables, lengths, q, k, v, f.float()), lambda: call(kp, vp, tables, lengths, q, k, v, profk.rotary_frequencies(66)),
           lambda: call(kp, vp, tables, lengths, q, k, v, f, starts=starts[:2]), lambda: call(kp, vp, tables, lengths, q, k, v, f, starts=starts.long()),
           lambda: call(kp, vp, tables, lengths, q, k, v, f, positions=lengths), lambda: call(kp, vp, tables, lengths, q, k, v, f, positions=lengths.long()[:1]),
           lambda: call(kp, vp, tables, lengths, q, k[:1], v[:1], f), lambda: call(kp, vp, tables, lengths, q, k, v, f, magnitude=float("nan")),
           lambda: call(kp, vp, tables, lengths, q, k.clone().requires_grad_(True), v, f), lambda: call(kp, vp, tables, lengths, q.clone().requires_grad_(True), k, v, f),
           lambda: call(kp, vp, tables, lengths, q, k, v.cpu(), f), lambda: call(kp, vp, tables, lengths, "q", k, v, f)]
    for n, f_ in enumerate(bad):
        with pytest.raises(profk.ProfkError):
            f_()
            pytest.fail(f"call {n} was not refused")
    assert torch.equal(kp, before)
