"""Values that are not finite in the cache under the attention of a chunk of new tokens: who does not see them has the same bits
as without them, whatever the pages' size (pages with a factor of eight tokens are copied by tile, others token by token)."""
import numpy as np
import pytest
import torch

import paper_2608_12573_b200 as profk
from paper_2608_12573_b200 import _build

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    _build.build()
    profk.lib()
    torch.cuda.set_device(0)


def _case(lengths, news, heads, kv_heads, dim, page, seed=0, dtype=torch.bfloat16):
    """q (rows, heads, dim), k, v, tables (pages in order), lengths, starts."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    need = [-(-n // page) for n in lengths]
    tables = torch.full((len(lengths), max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        tables[i, :n] = torch.arange(at, at + n, device="cuda")
        at += n
    k, v = (torch.randn(at, kv_heads, page, dim, generator=g, device="cuda").to(dtype) for _ in range(2))
    q = torch.randn(sum(news), heads, dim, generator=g, device="cuda").to(dtype)
    starts = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32, device="cuda")
    return q, k, v, tables, torch.tensor(lengths, dtype=torch.int32, device="cuda"), starts


def _call(q, k, v, tables, lengths, starts):
    return profk.paged_attention_chunk(q, k, v, tables, lengths, starts=starts)


@pytest.mark.parametrize("page", [1, 7, 12, 16, 100])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
def test_unseen_values_in_any_column(dim, page):
    lengths, news = [50, 19, 300, 700], [20, 19, 200, 260]
    case = _case(lengths, news, 4, 2, dim, page, seed=dim + page)
    q, k, v, tables, _, starts = case
    want = _call(*case)
    columns = sorted({3, min(70, dim - 9), dim // 2 + 1, dim - 1})
    for bad in (NAN, INF):
        k2, v2 = k.clone(), v.clone()
        for i, n in enumerate(lengths):
            if n % page:                                         # behind the last token: seen by no row
                k2[int(tables[i, n // page]), :, n % page:], v2[int(tables[i, n // page]), :, n % page:] = NAN, bad
        for _ in range(3):
            got = _call(q, k2, v2, *case[3:])
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            again = _call(*case)                                 # (what the calls before left in shared memory does not matter)
            assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])
        # one token near the end of each sequence, a column at a time: the rows in front of it know nothing of it
        for column in columns:
            v3 = v2.clone()
            for n, i in zip(lengths, range(4)):
                v3[int(tables[i, (n - 9) // page]), :, (n - 9) % page, column] = bad
            vector = [d for d in range(dim) if d // 8 == column // 8]
            rest = [d for d in range(dim) if d // 8 != column // 8]
            for _ in range(3):
                got = _call(q, k2, v3, *case[3:])
                assert torch.equal(got[1], want[1])
                for i in range(4):
                    a, z = int(starts[i]), int(starts[i + 1])
                    first = max(a, z - 9)
                    assert torch.equal(got[0][a:first], want[0][a:first]), (column, i)
                    assert torch.equal(got[0][first:z][..., rest], want[0][first:z][..., rest]), (column, i)
                    assert not torch.isfinite(got[0][first:z, :, column]).any(), (column, i)
                    # (the vector's other elements were left out of the product and added in fp32: they differ by the rounding of a weight,
                    # 2^-8 of at most |v| < 8, and half a step of the output)
                    near = [d for d in vector if d != column]
                    assert torch.allclose(got[0][first:z][..., near].float(), want[0][first:z][..., near].float(), rtol=2.0 ** -7, atol=2.0 ** -5)


@pytest.mark.parametrize("page", [7, 16])
@pytest.mark.parametrize("dim", [64, 128])
def test_long_items_with_many_bad_tokens_among_short_ones(dim, page):
    """The second half of an item's rows see many tokens with values that are not finite, which takes long, and short items follow
    that need the first half's warps only: what was noted for the long item has to outlast them."""
    lengths = [200, 20, 9, 20, 3] * 592
    case = _case(lengths, lengths, 1, 1, dim, page, seed=page)
    q, k, v, tables, _, starts = case
    want = _call(*case)
    bad = v.clone()
    first = 130
    long = tables[::5]
    for token in range(first, 200):
        bad[long[:, token // page].long(), 0, token % page, dim - 3] = NAN
    for _ in range(3):
        got = _call(q, k, bad, *case[3:])
        out, fine = got[0].view(592, -1, dim), want[0].view(592, -1, dim)
        assert torch.equal(got[1], want[1])
        assert torch.equal(out[:, :first], fine[:, :first]) and torch.equal(out[:, 200:], fine[:, 200:])
        assert torch.isnan(out[:, first:200, dim - 3]).all() and torch.equal(out[:, first:200, :dim - 8], fine[:, first:200, :dim - 8])
