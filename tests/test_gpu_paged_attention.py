"""Attention of one token over a paged cache against the 64-bit oracle on a GPU.

Tolerances.  A score is a sum of dim products that the matrix unit adds in fp32, at worst with one unit of the last place
lost per step: scale * sum |q k| * 2^-20 absolute, which moves a probability by as much relatively; the exponential and its
argument add 2^-22 + 2^-22 |y| (|y| <= 64 where it matters: 2^-16), the split of the probabilities into two numbers of the
cache's type leaves 2^-16.  An output entry may then be off by sum p |v| times twice the sum of these, plus half a unit in
the last place of its type; lse by the scores' error, 2^-16 and 2^-22 of itself."""
import numpy as np
import pytest
import torch

import paper_2608_12573_b200 as profk
from oracle import decode as oracle
from paper_2608_12573_b200 import _build

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    _build.build()
    profk.lib()
    torch.cuda.set_device(0)


def _case(lengths, heads, kv_heads, dim, page, dtype, seed=0, tokens_first=False, spare=3):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    tables = torch.full((len(lengths), max(need + [1])), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        tables[i, :n] = order[at:at + n]
        at += n
    shape = (pages, page, kv_heads, dim) if tokens_first else (pages, kv_heads, page, dim)
    k, v = (torch.randn(shape, generator=g, device="cuda").to(DTYPES[dtype]) for _ in range(2))
    if tokens_first:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    q = (torch.randn(len(lengths), heads, dim, generator=g, device="cuda") * 1.5).to(DTYPES[dtype])
    return q, k, v, tables, torch.tensor(lengths, dtype=torch.int32, device="cuda")


def _check(q, k, v, tables, lengths, scale=None, result=None):
    out, lse = profk.paged_attention(q, k, v, tables, lengths, scale) if result is None else result
    torch.cuda.synchronize()
    scale = q.shape[2] ** -0.5 if scale is None else scale
    host = [x.float().cpu().numpy() for x in (q, k, v)]
    t, n = tables.cpu().numpy(), lengths.cpu().numpy()
    want, want_lse = oracle.paged_attention(*host, t, n, scale)
    size, _ = oracle.paged_attention(host[0], host[1], np.abs(host[2]), t, n, scale)          # sum p |v|
    reach = np.zeros(want_lse.shape)                                                          # largest scale * sum |q k|
    group = q.shape[1] // k.shape[1]
    held = {}
    for s in range(len(n)):
        ids = [p for p in t[s][:-(-int(max(0, min(n[s], t.shape[1] * k.shape[2]))) // k.shape[2])] if 0 <= p < k.shape[0]]
        for h in range(q.shape[1]):
            if ids:
                held[s] = ids
                reach[s, h] = (np.abs(host[1][ids, h // group]).astype(np.float64) @ np.abs(host[0][s, h])).max() * scale
    rel = 2 * (reach * 2.0 ** -20 + 2.0 ** -16 + 2.0 ** -16)
    got, ulp = out.float().cpu().numpy().astype(np.float64), torch.finfo(q.dtype).eps
    off = np.abs(got - want)
    allowed = 0.5 * ulp * np.abs(want) + size * rel[..., None] + torch.finfo(q.dtype).tiny
    assert (off <= allowed).all(), f"out: {off.max()} at {np.unravel_index((off - allowed).argmax(), off.shape)}"
    got_lse = lse.cpu().numpy().astype(np.float64)
    empty = np.isneginf(want_lse)
    assert (np.isneginf(got_lse) == empty).all()
    off = np.abs(np.where(empty, 0, got_lse) - np.where(empty, 0, want_lse))
    assert (off <= reach * 2.0 ** -20 + 2.0 ** -16 + 2.0 ** -22 * np.abs(np.where(empty, 0, want_lse))).all(), f"lse: {off.max()}"
    return out, lse


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("dim", [8, 64, 72, 96, 128, 136, 256])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 2), (5, 1)])
def test_dims_and_heads(dtype, dim, heads, kv_heads):
    _check(*_case([1, 77, 300], heads, kv_heads, dim, 16, dtype, seed=dim + heads))


@pytest.mark.parametrize("heads,kv_heads", [(16, 1), (17, 1), (20, 1), (34, 2), (48, 3), (64, 1), (32, 32)])
def test_groups_of_any_size(heads, kv_heads):
    _check(*_case([130, 63], heads, kv_heads, 128, 32, "bf16", seed=heads))


@pytest.mark.parametrize("page", [1, 7, 16, 24, 64, 100, 256])
@pytest.mark.parametrize("tokens_first", [False, True])
def test_page_sizes_and_layouts(page, tokens_first):
    _check(*_case([1, 15, 16, 17, 63, 64, 65, 129, 500], 8, 2, 64, page, "f16", seed=page, tokens_first=tokens_first))


@pytest.mark.parametrize("lengths", [[0], [1], [0, 0, 0], [0, 5, 0, 0, 700, 0], [4000], [1] * 300, list(range(0, 200, 3)), [3000, 1, 2, 9, 2500]])
def test_lengths(lengths):
    out, lse = _check(*_case(lengths, 4, 2, 128, 16, "bf16", seed=len(lengths)))
    for i, n in enumerate(lengths):
        if n == 0:
            assert (out[i] == 0).all() and (lse[i] == -float("inf")).all()


def test_one_long_sequence_shared_by_all_ctas():
    q, k, v, tables, lengths = _case([60001], 8, 1, 128, 64, "bf16", seed=3)
    _check(q, k, v, tables, lengths)
    q[:, 0] = k[int(tables[0, 500]), 0, 3] * 4          # one token that takes nearly all the weight of head 0
    _check(q, k, v, tables, lengths)


def test_scores_that_rise_and_fall_far():
    q, k, v, tables, lengths = _case([900, 901], 2, 2, 64, 16, "bf16", seed=4)
    k *= torch.linspace(0.1, 12, 16, device="cuda").view(1, 1, 16, 1).to(k.dtype)
    _check(q * 2, k, v, tables, lengths, scale=0.3)


def test_pages_that_are_not_there():
    q, k, v, tables, lengths = _case([100, 64, 200], 4, 2, 64, 16, "bf16", seed=5)
    tables[0, 2] = -1
    tables[1, :] = -7
    tables[2, 5] = k.shape[0]
    out, lse = _check(q, k, v, tables, lengths)
    assert (out[1] == 0).all() and torch.isneginf(lse[1]).all()


def test_lengths_outside_the_table_are_taken_into_it():
    q, k, v, tables, lengths = _case([64, 64], 4, 2, 64, 16, "f16", seed=6)
    want = profk.paged_attention(q, k, v, tables, lengths)
    lengths[0], lengths[1] = 1 << 30, -5
    got = profk.paged_attention(q, k, v, tables, lengths)
    assert torch.equal(got[0][0], want[0][0]) and (got[0][1] == 0).all()


def test_what_lies_behind_a_sequence_does_not_matter():
    q, k, v, tables, lengths = _case([50, 19], 4, 2, 96, 16, "bf16", seed=7)
    want = profk.paged_attention(q, k, v, tables, lengths)
    for i, n in enumerate([50, 19]):
        k[int(tables[i, n // 16]), :, n % 16:] = float("nan")
        v[int(tables[i, n // 16]), :, n % 16:] = float("inf")
    unused = [p for p in range(k.shape[0]) if p not in tables.flatten().tolist()]
    k[unused], v[unused] = float("nan"), float("nan")
    got = profk.paged_attention(q, k, v, tables, lengths)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_offsets_that_pass_32_bits():
    """A cache of 4.3 GB whose last pages lie behind 2^31 elements."""
    pages, page, dim = 17000, 256, 256
    k = torch.zeros(pages, 2, page, dim, dtype=torch.float16, device="cuda")
    assert k.numel() > 1 << 31
    at = [pages - 1, 3, pages - 2]
    k[at] = torch.randn(3, 2, page, dim, device="cuda").half()
    v = k
    q = torch.randn(1, 2, dim, device="cuda").half()
    tables = torch.tensor([at], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([700], dtype=torch.int32, device="cuda")
    out, lse = profk.paged_attention(q, k, v, tables, lengths)
    small = k[at].contiguous()
    _check(q, small, small, torch.tensor([[0, 1, 2]], dtype=torch.int32, device="cuda"), lengths, result=(out, lse))


def test_strides():
    q, k, v, tables, lengths = _case([100, 33], 6, 3, 64, 16, "bf16", seed=8)
    want = profk.paged_attention(q, k, v, tables, lengths)
    wide_q = torch.zeros(2, 9, 80, dtype=q.dtype, device="cuda")
    wide_q[:, 1:7, 2:66] = q
    both = torch.zeros(k.shape[0], 2, 3, 16, 72, dtype=k.dtype, device="cuda")          # keys beside values, padded rows
    both[:, 0, ..., 8:], both[:, 1, ..., :64] = k, v
    wide_t = torch.full((2, tables.shape[1] + 5), 1 << 29, dtype=torch.int32, device="cuda")
    wide_t[:, :tables.shape[1]] = tables
    got = profk.paged_attention(wide_q[:, 1:7, 2:66], both[:, 0, ..., 8:], both[:, 1, ..., :64], wide_t[:, :tables.shape[1]], lengths)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_the_same_call_gives_the_same_bits_on_any_stream_and_in_a_graph():
    q, k, v, tables, lengths = _case([5000, 3, 0, 1200, 77], 16, 2, 128, 16, "bf16", seed=9)
    want = _check(q, k, v, tables, lengths)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = profk.paged_attention(q.clone(), k, v, tables, lengths)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = profk.paged_attention(q, k, v, tables, lengths)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_refusals():
    q, k, v, tables, lengths = _case([40, 20], 4, 2, 64, 16, "bf16")
    call = profk.paged_attention
    bad = [lambda: call(q.float(), k.float(), v.float(), tables, lengths), lambda: call(q, k.half(), v.half(), tables, lengths),
           lambda: call(q[:, :3], k, v, tables, lengths), lambda: call(q, k, v[:-1], tables, lengths), lambda: call(q, k, v, tables.long(), lengths),
           lambda: call(q, k, v, tables, lengths.long()), lambda: call(q[:1], k, v, tables, lengths), lambda: call(q, k, v, tables, lengths[:1]),
           lambda: call(q[..., :32], k, v, tables, lengths), lambda: call(q[..., :60], k[..., :60], v[..., :60], tables, lengths),
           lambda: call(q, k, v, tables, lengths, scale=0.0), lambda: call(q, k, v, tables, lengths, scale=-1.0),
           lambda: call(q, k, v, tables, lengths, scale=float("nan")), lambda: call(q.cpu(), k, v, tables, lengths),
           lambda: call(q, k, v, tables[:, :0], lengths), lambda: call(q[..., ::2], k[..., ::2], v[..., ::2], tables, lengths),
           lambda: call(torch.zeros(2, 2, 264, dtype=q.dtype, device="cuda"), torch.zeros(4, 2, 16, 264, dtype=q.dtype, device="cuda"),
                        torch.zeros(4, 2, 16, 264, dtype=q.dtype, device="cuda"), tables, lengths),
           lambda: call(q[..., :56], k[..., 4:60], v[..., 4:60], tables, lengths)]
    for n, f in enumerate(bad):
        with pytest.raises(profk.ProfkError):
            f()
            pytest.fail(f"call {n} was not refused")
    _check(q, k, v, tables, lengths)
