"""Attention of a chunk of new tokens over a paged cache against the 64-bit oracle on a GPU.

Tolerances.  A score is a sum of dim products that the matrix unit adds in fp32, at worst with one unit of the last place
lost per step: scale * sum |q k| * 2^-20 absolute, which moves a weight by as much relatively; the exponential and its
argument add 2^-22 + 2^-22 |y| (|y| <= 64 where it matters: 2^-16).  A weight is rounded once to the cache's type: half a step,
eps / 2 of it (fp16: 2^-36 of the largest, too: half a subnormal step, 2^-25, of weights that are lifted by 2^11).  The sum over n tokens is taken in steps of 16, each off by
2^-23 of what it has at worst.  So an output entry may be off by sum p |v| times eps / 2 + n / 16 * 2^-23 + twice the first two, plus
half a unit in the last place of its type; lse by the scores' error, 2^-16 and 2^-22 of itself."""
import numpy as np
import pytest
import torch

import paper_2608_12573_b200 as profk
from oracle import prompt as oracle
from paper_2608_12573_b200 import _build

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    _build.build()
    profk.lib()
    torch.cuda.set_device(0)


def _case(lengths, news, heads, kv_heads, dim, page, dtype, seed=0, tokens_first=False, spare=3, behind=0):
    """q (rows, heads, dim), k, v, tables, lengths, starts; `behind` rows that no sequence holds."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    need = [-(-max(n, 0) // page) for n in lengths]
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
    q = (torch.randn(sum(news) + behind, heads, dim, generator=g, device="cuda") * 1.5).to(DTYPES[dtype])
    starts = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32, device="cuda")
    return q, k, v, tables, torch.tensor(lengths, dtype=torch.int32, device="cuda"), starts


def _check(q, k, v, tables, lengths, starts, scale=None, result=None):
    out, lse = profk.paged_attention_chunk(q, k, v, tables, lengths, starts=starts, scale=scale) if result is None else result
    torch.cuda.synchronize()
    scale = q.shape[2] ** -0.5 if scale is None else scale
    host = [x.float().cpu().numpy() for x in (q, k, v)]
    want, want_lse, size, reach = oracle.paged_attention_chunk(*host, tables.cpu().numpy(), lengths.cpu().numpy(), scale, starts.cpu().numpy())
    eps = torch.finfo(q.dtype).eps / 2
    rel = eps + max(0, int(lengths.max())) / 16 * 2.0 ** -23 + 2 * (reach * 2.0 ** -20 + 2.0 ** -16)
    got = out.double().cpu().numpy()
    fine = np.isfinite(want)
    assert (np.isfinite(got) == fine).all(), "values that are not finite"
    off = np.abs(np.where(fine, got, 0) - np.where(fine, want, 0))
    tiny = torch.finfo(q.dtype).tiny + (2.0 ** -36 * int(lengths.max()) * 8 if q.dtype == torch.float16 else 0)
    allowed = eps * np.abs(np.where(fine, want, 0)) + np.where(fine, size, 0) * rel[..., None] + tiny
    assert (off <= allowed).all(), f"out: {off.max()} (allowed {allowed.flat[(off - allowed).argmax()]}) at {np.unravel_index((off - allowed).argmax(), off.shape)}"
    got_lse = lse.double().cpu().numpy()
    empty = np.isneginf(want_lse)
    assert (np.isneginf(got_lse) == empty).all()
    off = np.abs(np.where(empty, 0, got_lse) - np.where(empty, 0, want_lse))
    assert (off <= reach * 2.0 ** -20 + 2.0 ** -16 + 2.0 ** -22 * np.abs(np.where(empty, 0, want_lse))).all(), f"lse: {off.max()}"
    return out, lse


def test_one_tile():
    _check(*_case([20], [20], 1, 1, 64, 16, "bf16"))
    _check(*_case([20], [20], 1, 1, 128, 16, "bf16"))
    _check(*_case([20], [20], 1, 1, 256, 16, "bf16"))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("dim", [8, 64, 72, 96, 128, 136, 256])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 2), (5, 1)])
def test_dims_and_heads(dtype, dim, heads, kv_heads):
    _check(*_case([1, 77, 300, 290], [1, 5, 300, 130], heads, kv_heads, dim, 16, dtype, seed=dim + heads))


@pytest.mark.parametrize("heads,kv_heads", [(16, 1), (17, 1), (34, 2), (48, 3), (64, 1), (200, 1), (300, 1), (32, 32)])
def test_groups_of_any_size(heads, kv_heads):
    _check(*_case([130, 63, 40], [7, 63, 1], heads, kv_heads, 128, 32, "bf16", seed=heads))


@pytest.mark.parametrize("page", [1, 7, 16, 24, 64, 100, 256])
@pytest.mark.parametrize("tokens_first", [False, True])
def test_page_sizes_and_layouts(page, tokens_first):
    lengths = [1, 15, 16, 17, 63, 64, 65, 129, 500]
    _check(*_case(lengths, [1, 15, 3, 17, 60, 1, 2, 100, 300], 8, 2, 64, page, "f16", seed=page, tokens_first=tokens_first))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("lengths,news", [([0], [0]), ([5], [0]), ([1], [1]), ([0, 5, 0, 700, 0], [0, 5, 0, 300, 0]), ([4000], [1]), ([4000], [400]), ([1] * 300, [1] * 300),
                                          (list(range(0, 200, 3)), [n // 2 for n in range(0, 200, 3)]), ([127, 128, 129, 255, 256, 257], [127, 128, 129, 255, 256, 257]),
                                          ([383, 384, 385, 513], [2, 129, 256, 257])])
def test_lengths(dim, lengths, news):
    _check(*_case(lengths, news, 4, 2, dim, 16, "bf16", seed=len(lengths), behind=2))


def test_more_new_tokens_than_there_are():
    """Lengths below the number of new tokens, negative ones and such that pass the table's end."""
    q, k, v, tables, lengths, starts = _case([64, 64, 64, 64, 64], [10, 64, 40, 20, 30], 4, 2, 64, 16, "bf16", seed=6)
    lengths.copy_(torch.tensor([4, 30, -50, 70, 1 << 30]))
    out, lse = _check(q, k, v, tables, lengths, starts)
    assert (out[:6] == 0).all() and torch.isneginf(lse[:6]).all() and (out[74:114] == 0).all()
    lengths.fill_(-(2 ** 31))
    out, lse = profk.paged_attention_chunk(q, k, v, tables, lengths, starts=starts)
    assert (out == 0).all() and torch.isneginf(lse).all()


def test_rows_that_no_sequence_holds():
    q, k, v, tables, lengths, starts = _case([50, 60], [20, 30], 4, 2, 64, 16, "bf16", behind=40)
    starts += 7
    out, lse = _check(q, k, v, tables, lengths, starts)
    for rows in (slice(0, 7), slice(57, 90)):
        assert (out[rows] == 0).all() and torch.isneginf(lse[rows]).all()


def test_one_long_sequence_shared_by_all_ctas():
    for news in ([3], [200]):
        q, k, v, tables, lengths, starts = _case([30001], news, 8, 1, 128, 64, "bf16", seed=3)
        _check(q, k, v, tables, lengths, starts)
        q[:, 0] = k[int(tables[0, 300]), 0, 3] * 4       # one token that takes nearly all the weight of head 0
        _check(q, k, v, tables, lengths, starts)


@pytest.mark.parametrize("dim,heads", [(64, 40), (128, 40), (256, 20)])
def test_many_items_of_many_tiles_to_a_cta(dim, heads):
    """Items whose tiles are taken in another order than they lie in, with tokens at the end that only some rows see."""
    q, k, v, tables, lengths, starts = _case([4400, 4600, 4300], [300, 260, 513], heads, heads, dim, 32, "bf16", seed=dim)
    want = profk.paged_attention_chunk(q, k, v, tables, lengths, starts=starts)
    some = [0, 1, heads // 2, heads - 1]                 # (the oracle's time: a few of the heads)
    _check(q[:, some], k[:, some], v[:, some], tables, lengths, starts, result=(want[0][:, some], want[1][:, some]))
    for i, n in enumerate([4400, 4600, 4300]):
        v[int(tables[i, (n - 9) // 32]), :, (n - 9) % 32, 3] = float("nan")
    got = profk.paged_attention_chunk(q, k, v, tables, lengths, starts=starts)
    for i in range(3):
        a, z = int(starts[i]), int(starts[i + 1])
        assert torch.equal(got[0][a:z - 9], want[0][a:z - 9]) and torch.isnan(got[0][z - 9:z, :, 3]).all() and torch.equal(got[0][z - 9:z, :, 8:], want[0][z - 9:z, :, 8:])


def test_scores_that_rise_and_fall_far():
    for dim in (64, 128, 256):
        for dtype in DTYPES:
            q, k, v, tables, lengths, starts = _case([900, 901, 300], [4, 500, 300], 2, 2, dim, 16, dtype, seed=4)
            k *= torch.linspace(0.1, 12, 16, device="cuda").view(1, 1, 16, 1).to(k.dtype)
            _check(q * 2, k, v, tables, lengths, starts, scale=0.3 * 8 / dim ** 0.5)


def test_small_weights_beside_a_sink():
    """One token with nearly all the weight and values of zero: the others' share, 2^-20 each in fp16 and bf16 alike, is kept."""
    for dtype in DTYPES:
        q, k, v, tables, lengths, starts = _case([700], [5], 2, 2, 64, 16, dtype, seed=11)
        q.zero_(), k.zero_()
        q[..., 0] = 1.0
        k[int(tables[0, 0]), :, 3, 0], v[int(tables[0, 0]), :, 3] = 14.0, 0.0
        v.abs_()
        _check(q, k, v, tables, lengths, starts, scale=1.0)


def test_pages_that_are_not_there():
    q, k, v, tables, lengths, starts = _case([100, 64, 200, 600], [50, 64, 3, 400], 4, 2, 64, 16, "bf16", seed=5)
    tables[0, 2] = -1
    tables[1, :] = -7
    tables[2, 5] = k.shape[0]
    tables[3, 3:30] = -1
    out, lse = _check(q, k, v, tables, lengths, starts)
    assert (out[50:114] == 0).all() and torch.isneginf(lse[50:114]).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_what_a_row_does_not_see_does_not_reach_it(dim):
    q, k, v, tables, lengths, starts = _case([50, 19, 300], [20, 19, 200], 4, 2, dim, 16, "bf16", seed=7)
    want = profk.paged_attention_chunk(q, k, v, tables, lengths, starts=starts)
    for i, n in enumerate([50, 19, 300]):
        if n % 16:
            k[int(tables[i, n // 16]), :, n % 16:], v[int(tables[i, n // 16]), :, n % 16:] = float("nan"), float("inf")
    unused = [p for p in range(k.shape[0]) if p not in tables.flatten().tolist()]
    k[unused], v[unused] = float("nan"), float("nan")
    got = profk.paged_attention_chunk(q, k, v, tables, lengths, starts=starts)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # the last tokens of each sequence: only the rows at and behind them may know
    for bad in (float("nan"), float("inf")):
        k2, v2 = k.clone(), v.clone()
        hit = []
        for i, (n, new) in enumerate(zip([50, 19, 300], [20, 19, 200])):
            for back in (1, 4, 11):
                at = n - back
                v2[int(tables[i, at // 16]), 1, at % 16, dim // 2] = bad
                if back == 1:
                    k2[int(tables[i, at // 16]), 0, at % 16, 1] = float("nan")
            hit.append(n - 11)
        got = profk.paged_attention_chunk(q, k2, v2, tables, lengths, starts=starts)
        for i, (n, new) in enumerate(zip([50, 19, 300], [20, 19, 200])):
            a, z = int(starts[i]), int(starts[i + 1])
            first_bad = a + hit[i] - (n - new)
            assert torch.equal(got[0][a:z - 1, :2], want[0][a:z - 1, :2]) and torch.isnan(got[0][z - 1, :2]).all()        # head 0's keys
            assert torch.equal(got[0][a:first_bad, 2:], want[0][a:first_bad, 2:])
            touched = got[0][first_bad:z, 2:, dim // 2]
            assert (torch.isnan(touched) if bad != bad else ~torch.isfinite(touched)).all()
            rest = [d for d in range(dim) if d // 8 != dim // 2 // 8]
            assert torch.equal(got[0][a:z, 2:][..., rest], want[0][a:z, 2:][..., rest])
            # the other elements of the vectors that were taken out come back to within the rounding of the weights
            near = [d for d in range(dim) if d // 8 == dim // 2 // 8 and d != dim // 2]
            assert torch.allclose(got[0][a:z, 2:][..., near].float(), want[0][a:z, 2:][..., near].float(), rtol=2.0 ** -7, atol=2.0 ** -7)


def test_values_that_are_not_finite_are_seen():
    q, k, v, tables, lengths, starts = _case([700], [300], 2, 1, 128, 16, "bf16", seed=17)
    v[int(tables[0, 2]), 0, 3, 5] = float("inf")         # every row sees it
    out, _ = profk.paged_attention_chunk(q, k, v, tables, lengths, starts=starts)
    assert (~torch.isfinite(out[..., 5])).all() and torch.isfinite(out[..., :5]).all() and torch.isfinite(out[..., 6:]).all()


def test_offsets_that_pass_32_bits():
    """A cache of 4.3 GB whose last pages lie behind 2^31 elements."""
    pages, page, dim = 17000, 256, 256
    k = torch.zeros(pages, 2, page, dim, dtype=torch.float16, device="cuda")
    assert k.numel() > 1 << 31
    at = [pages - 1, 3, pages - 2]
    k[at] = torch.randn(3, 2, page, dim, device="cuda").half()
    q = torch.randn(40, 2, dim, device="cuda").half()
    tables = torch.tensor([at], dtype=torch.int32, device="cuda")
    lengths, starts = torch.tensor([700], dtype=torch.int32, device="cuda"), torch.tensor([0, 40], dtype=torch.int32, device="cuda")
    result = profk.paged_attention_chunk(q, k, k, tables, lengths, starts=starts)
    small = k[at].contiguous()
    _check(q, small, small, torch.tensor([[0, 1, 2]], dtype=torch.int32, device="cuda"), lengths, starts, result=result)


def test_strides():
    q, k, v, tables, lengths, starts = _case([100, 33], [50, 33], 6, 3, 64, 16, "bf16", seed=8)
    want = profk.paged_attention_chunk(q, k, v, tables, lengths, starts=starts)
    both = torch.zeros(k.shape[0], 2, 3, 16, 72, dtype=k.dtype, device="cuda")          # keys beside values, padded rows
    both[:, 0, ..., 8:], both[:, 1, ..., :64] = k, v
    wide_t = torch.full((2, tables.shape[1] + 5), 1 << 29, dtype=torch.int32, device="cuda")
    wide_t[:, :tables.shape[1]] = tables
    for shift in (0, 1, 2, 8):                           # queries at any alignment
        wide_q = torch.zeros(83, 9, 80, dtype=q.dtype, device="cuda")
        wide_q[:, 1:7, shift:shift + 64] = q
        got = profk.paged_attention_chunk(wide_q[:, 1:7, shift:shift + 64], both[:, 0, ..., 8:], both[:, 1, ..., :64], wide_t[:, :tables.shape[1]], lengths, starts=starts)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    by_head = q.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(profk.paged_attention_chunk(by_head, k, v, tables, lengths, starts=starts)[0], want[0])


def test_even_chunks_are_ragged_ones():
    q, k, v, tables, lengths, starts = _case([100, 33, 40], [30, 30, 30], 6, 3, 64, 16, "bf16", seed=8)
    want = _check(q, k, v, tables, lengths, starts)
    got = profk.paged_attention_chunk(q.view(3, 30, 6, 64), k, v, tables, lengths)
    assert got[0].shape == (3, 30, 6, 64) and got[1].shape == (3, 30, 6)
    assert torch.equal(got[0].flatten(0, 1), want[0]) and torch.equal(got[1].flatten(0, 1), want[1])
    swapped = q.view(3, 30, 6, 64).transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(profk.paged_attention_chunk(swapped, k, v, tables, lengths)[0], got[0])
    assert profk.paged_attention_chunk(q.view(3, 30, 6, 64)[:, :0], k, v, tables, lengths)[0].shape == (3, 0, 6, 64)


def test_one_token_at_a_time_is_the_form_for_one_token():
    q, k, v, tables, lengths, starts = _case([100, 333, 40], [1, 1, 1], 8, 2, 128, 16, "bf16", seed=9)
    out, lse = _check(q, k, v, tables, lengths, starts)
    one = profk.paged_attention(q, k, v, tables, lengths)
    assert torch.allclose(out.float(), one[0].float(), rtol=2.0 ** -7, atol=2.0 ** -7) and torch.allclose(lse, one[1], rtol=2.0 ** -20, atol=2.0 ** -14)


def test_the_same_call_gives_the_same_bits_on_any_stream_and_in_a_graph():
    q, k, v, tables, lengths, starts = _case([5000, 3, 0, 1200, 77], [300, 3, 0, 4, 77], 16, 2, 128, 16, "bf16", seed=9)
    want = _check(q, k, v, tables, lengths, starts)
    for _ in range(5):
        got = profk.paged_attention_chunk(q, k, v, tables, lengths, starts=starts)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = profk.paged_attention_chunk(q.clone(), k, v, tables, lengths, starts=starts)
    here = profk.paged_attention_chunk(q, k, v, tables, lengths, starts=starts)          # (two calls at once)
    torch.cuda.current_stream().wait_stream(side)
    for r in (got, here):
        assert torch.equal(r[0], want[0]) and torch.equal(r[1], want[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = profk.paged_attention_chunk(q, k, v, tables, lengths, starts=starts)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_broadcast_queries_and_heads():
    q, k, v, tables, lengths, starts = _case([100, 33], [50, 33], 6, 3, 64, 16, "bf16", seed=8)
    _check(q[:, :1].expand(83, 6, 64), k, v, tables, lengths, starts)
    _check(q, k[:, :1].expand(-1, 3, -1, -1), v[:, :1].expand(-1, 3, -1, -1), tables, lengths, starts)


def test_many_sequences():
    lengths = [(i * 7) % 40 + 1 for i in range(5000)]
    _check(*_case(lengths, [min(n, i % 3 + 1) for i, n in enumerate(lengths)], 2, 1, 64, 8, "bf16", seed=4))


@pytest.mark.parametrize("starts", [[5, -7, 1000, 93], [93, 50, 20, 0], [-2 ** 31, 2 ** 31 - 1, -1, 7], [0, 93, 0, 93]])
def test_starts_that_are_none_stay_in_bounds(starts):
    q, k, v, tables, lengths, _ = _case([100, 33, 60], [50, 33, 10], 6, 3, 64, 16, "bf16", seed=8)
    fenced = torch.full((95, 6, 64), 7.0, dtype=q.dtype, device="cuda")
    fenced[1:94] = q
    out, lse = profk.paged_attention_chunk(fenced[1:94], k, v, tables, lengths, starts=torch.tensor(starts, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert out.shape == q.shape and lse.shape == (93, 6) and (fenced[0] == 7).all() and (fenced[94] == 7).all()


def test_calls_at_once_and_two_graphs():
    cases = [_case([3000, 20, 700], [300, 20, 4], 16, 4, 128, 16, "bf16", seed=1), _case([900, 1000], [100, 1000], 4, 4, 64, 32, "f16", seed=2),
             _case([500], [200], 4, 2, 256, 8, "bf16", seed=3)]
    call = lambda c: profk.paged_attention_chunk(*c[:5], starts=c[5])  # noqa: E731
    want = [call(c) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        got = []
        for stream, c in zip(streams, cases):
            with torch.cuda.stream(stream):
                got.append(call(c))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))
    graphs = []
    for c in cases:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            result = call(c)
        graphs.append((graph, result))
    for _ in range(3):
        for graph, _ in graphs:
            graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for (_, g), w in zip(graphs, want) for a, b in zip(g, w))


def test_refusals():
    q, k, v, tables, lengths, starts = _case([40, 20], [5, 7], 4, 2, 64, 16, "bf16")
    call = lambda *a, starts=starts, **how: profk.paged_attention_chunk(*a, starts=starts, **how)  # noqa: E731
    zeros = lambda *shape: torch.zeros(shape, dtype=q.dtype, device="cuda")  # noqa: E731
    bad = [lambda: call(q.float(), k.float(), v.float(), tables, lengths), lambda: call(q, k.half(), v.half(), tables, lengths), lambda: call(q[:, :3], k, v, tables, lengths),
           lambda: call(q, k, v[:-1], tables, lengths), lambda: call(q, k, v, tables.long(), lengths), lambda: call(q, k, v, tables, lengths.long()),
           lambda: call(q, k, v, tables, lengths[:1]), lambda: call(q[..., :32], k, v, tables, lengths), lambda: call(q[..., :60], k[..., :60], v[..., :60], tables, lengths),
           lambda: call(q, k, v, tables, lengths, scale=0.0), lambda: call(q, k, v, tables, lengths, scale=float("nan")), lambda: call(q.cpu(), k, v, tables, lengths),
           lambda: call(q, k, v, tables[:, :0], lengths), lambda: call(q[..., ::2], k[..., ::2], v[..., ::2], tables, lengths),
           lambda: call(zeros(12, 2, 264), zeros(4, 2, 16, 264), zeros(4, 2, 16, 264), tables, lengths), lambda: call(q[..., :56], k[..., 4:60], v[..., 4:60], tables, lengths),
           lambda: call(q, k, v, tables, lengths, starts=None), lambda: call(q[None], k, v, tables, lengths), lambda: call(q, k, v, tables, lengths, starts=starts[:2]),
           lambda: call(q, k, v, tables, lengths, starts=starts.long()), lambda: call(q, k, v, tables, lengths, starts=starts.cpu()),
           lambda: call(q.view(2, 6, 4, 64)[:1], k, v, tables, lengths, starts=None), lambda: call(q.clone().requires_grad_(True), k, v, tables, lengths),
           lambda: call(q, k.clone().requires_grad_(True), v, tables, lengths)]
    for n, f in enumerate(bad):
        with pytest.raises(profk.ProfkError):
            f()
            pytest.fail(f"call {n} was not refused")
    _check(q, k, v, tables, lengths, starts)
