"""Forking, growing, releasing, compacting, copying and appending pages, against the oracle on a GPU: whole numbers and moved
bits, compared exactly."""
import numpy as np
import pytest
import torch

import paper_2608_12573_b200 as profk
from oracle import decode as oracle
from paper_2608_12573_b200 import _build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    _build.build()
    profk.lib()
    torch.cuda.set_device(0)


def _int32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _pool(layers, pages, kv_heads, page, dim, seed, tokens_first=False):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    shape = (layers, 2, pages, page, kv_heads, dim) if tokens_first else (layers, 2, pages, kv_heads, page, dim)
    pool = torch.randint(-30000, 30000, shape, generator=g, device="cuda", dtype=torch.int16).view(torch.bfloat16)
    return pool.transpose(3, 4) if tokens_first else pool


def _state(lengths, page, width, pages, rng, shared=0):
    """Tables whose sequences share their first `shared` pages; the counts of their entries."""
    order = rng.permutation(pages)
    tables = np.full((len(lengths), width), -1, dtype=np.int32)
    at = shared
    for i, n in enumerate(lengths):
        need = -(-n // page)
        both = min(shared, n // page)
        tables[i, :both] = order[:both]
        tables[i, both:need] = order[at:at + need - both]
        at += need - both
    assert at <= pages
    refs = np.zeros(pages, dtype=np.int32)
    for t in tables[tables >= 0]:
        refs[t] += 1
    return tables, refs


def _host(pool):
    return pool.view(torch.int16).cpu().numpy().copy()


def _check_fork(pool, tables, lengths, refs, parents, grow, page):
    before = None if pool is None else _host(pool)
    got = profk.pages_fork(pool, _int32(tables).view(tables.shape), _int32(lengths), _int32(refs), _int32(parents), grow=grow,
                           page_size=None if pool is not None else page)
    torch.cuda.synchronize()
    stand_in = before if pool is not None else np.zeros((1, 2, len(refs), 1, page, 1), dtype=np.int16)
    want = oracle.fork(stand_in, tables, lengths, refs, parents, grow)
    np.testing.assert_array_equal(got.tables.cpu().numpy(), want[0])
    np.testing.assert_array_equal(got.lengths.cpu().numpy(), want[1])
    np.testing.assert_array_equal(got.refs.cpu().numpy(), want[2])
    assert int(got.missing) == want[3]
    if pool is not None:
        np.testing.assert_array_equal(_host(pool), before)
    return got, want


@pytest.mark.parametrize("page", [1, 5, 16, 64])
@pytest.mark.parametrize("tokens_first", [False, True])
@pytest.mark.parametrize("grow", [0, 1, 40])
def test_fork(page, tokens_first, grow):
    rng = np.random.default_rng(page + grow)
    lengths = np.array([0, 1, page, page + 1, 3 * page - 1, 100, 101])
    width = -(-(max(lengths) + grow) // page)
    tables, refs = _state(lengths, page, width, 400 + 16 * width, rng)
    pool = _pool(2, len(refs), 3, page, 24, 1, tokens_first)
    parents = np.array([5, 5, 1, -1, 3, 3, 3, 6, 99, 0, 4, 5])
    got, want = _check_fork(pool, tables, lengths, refs, parents, grow, page)
    # and on from there, into fewer sequences
    _check_fork(pool, want[0], want[1].astype(np.int64), want[2], np.array([11, 0, 0]), 1, page)


@pytest.mark.parametrize("n_old,n", [(1, 1), (1, 70), (70, 1), (300, 1500), (2500, 2500), (3, 0), (0, 4)])
def test_fork_counts_of_sequences(n_old, n):
    rng = np.random.default_rng(n_old)
    page, shared = 16, 2
    lengths = rng.integers(32, 90, n_old)
    tables, refs = _state(lengths, page, 7, 6 * n_old + 5 * n + 10, rng, shared)
    pool = _pool(1, len(refs), 1, page, 8, 2)
    parents = rng.integers(-1, max(1, n_old), n) if n_old else np.zeros(n, dtype=np.int64)
    _check_fork(pool, tables, lengths, refs, parents, 1, page)
    _check_fork(None, tables, lengths, refs, parents, 3, page)


def test_fork_without_enough_pages():
    rng = np.random.default_rng(3)
    lengths = np.array([20, 17, 33, 0])
    tables, refs = _state(lengths, 16, 4, 9, rng)
    pool = _pool(2, 9, 2, 16, 16, 3)
    for grow in (0, 13, 200):
        _check_fork(pool, tables, lengths, refs, np.array([0, 0, 2, 2, 1, 3, 0]), grow, 16)
    refs[:] = np.maximum(refs, 1)
    _check_fork(pool, tables, lengths, refs, np.array([0, 0, 1, 1]), 16, 16)
    # a page that is not there is neither copied nor counted
    tables[0, 1], tables[1, 0] = -1, 77
    refs[4] = 0
    _check_fork(pool, tables, lengths, refs, np.array([0, 0, 1, 1, 2]), 1, 16)


@pytest.mark.parametrize("pages", [1, 5000, 40001])
def test_fork_looks_for_free_pages_everywhere(pages):
    refs = np.ones(pages, dtype=np.int32)
    refs[-1:] = 0
    refs[pages // 3] = 0
    refs[pages // 2] = -2                                   # counts below zero are free too
    tables, lengths = np.full((2, 3), -1, dtype=np.int32), np.array([0, 0])
    _check_fork(None, tables, lengths, refs, np.array([0, 1, 1, 0]), 17, 16)


@pytest.mark.parametrize("pages,live", [(1, 1), (1, 0), (2, 1), (64, 64), (64, 0), (63, 31), (500, 450), (9001, 100)])
@pytest.mark.parametrize("tokens_first", [False, True])
def test_compact(pages, live, tokens_first):
    rng = np.random.default_rng(pages + live)
    refs = np.zeros(pages, dtype=np.int32)
    refs[rng.permutation(pages)[:live]] = rng.integers(1, 4, live)
    if pages > live:
        refs[np.flatnonzero(refs == 0)[0]] = -1
    tables = rng.integers(-1, pages + 1, (5, 40)).astype(np.int32)
    pool = _pool(2, pages, 2, 4, 8, 4, tokens_first)
    before = _host(pool)
    got = profk.pages_compact(pool, _int32(tables), _int32(refs))
    torch.cuda.synchronize()
    want = oracle.compact(before, tables, refs)
    for g, w in zip(got[:3], want[:3]):
        np.testing.assert_array_equal(g.cpu().numpy(), w)
    assert int(got.live) == want[3] == live
    np.testing.assert_array_equal(_host(pool), before)
    alone = profk.pages_compact(None, _int32(tables), _int32(refs))
    assert all(torch.equal(a, b) for a, b in zip(alone, got))


def test_copy():
    pool = _pool(3, 50, 2, 16, 40, 5)
    want = _host(pool)
    src, dst = [3, 9, -1, 4, 50, 7, 8], [10, 11, 12, -2, 13, 7, 49]
    for s, d in [(3, 10), (9, 11), (8, 49)]:
        want[:, :, d] = want[:, :, s]
    profk.pages_copy(pool, _int32(src), _int32(dst))
    np.testing.assert_array_equal(_host(pool), want)
    profk.pages_copy(pool, _int32([]), _int32([]))


@pytest.mark.parametrize("tokens", [1, 5])
@pytest.mark.parametrize("tokens_first", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.uint8])
def test_append(tokens, tokens_first, dtype):
    page, kv_heads, dim, lengths = 4, 3, 16, [1, 4, 5, 23, 0, 9]
    rng = np.random.default_rng(tokens)
    tables, refs = _state(lengths, page, 6, 40, rng)
    tables[5, 2] = -1
    shape = (40, page, kv_heads, dim) if tokens_first else (40, kv_heads, page, dim)
    k, v = torch.zeros(shape, dtype=dtype, device="cuda"), torch.zeros(shape, dtype=dtype, device="cuda")
    if tokens_first:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    new = torch.randint(1, 100, (2, 6, tokens, kv_heads, dim), device="cuda").to(dtype)
    want = [np.zeros((40, kv_heads, page, dim)) for _ in range(2)]
    host = new.float().cpu().numpy()
    for s, n in enumerate(lengths):
        for t in range(tokens):
            at = n - tokens + t
            if at >= 0 and tables[s, at // page] >= 0:
                for x in range(2):
                    want[x][tables[s, at // page], :, at % page] = host[x, s, t]
    args = (new[0, :, 0], new[1, :, 0]) if tokens == 1 else (new[0], new[1])
    profk.pages_append(k, v, _int32(tables), _int32(lengths), *args)
    np.testing.assert_array_equal(k.float().cpu().numpy(), want[0])
    np.testing.assert_array_equal(v.float().cpu().numpy(), want[1])


def test_in_a_graph_and_on_another_stream():
    rng = np.random.default_rng(6)
    lengths = np.array([20, 40, 50])
    tables, refs = _state(lengths, 16, 5, 60, rng)
    pool = _pool(2, 60, 2, 16, 32, 6)
    args = [_int32(tables), _int32(lengths), _int32(refs), _int32([0, 0, 1, 2, 2])]
    want = profk.pages_fork(pool, *args, grow=1)
    bits = _host(pool)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = profk.pages_fork(pool, *args, grow=1)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = profk.pages_fork(pool, *args, grow=1)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    np.testing.assert_array_equal(_host(pool), bits)


def test_refusals():
    pool = _pool(1, 20, 2, 16, 32, 7)
    t, n, r, p = _int32([[0, 1], [2, 3]]), _int32([20, 30]), _int32([1] * 4 + [0] * 16), _int32([0, 0])
    k = pool[0, 0]
    new = torch.zeros(2, 2, 32, dtype=pool.dtype, device="cuda")
    bad = [lambda: profk.pages_fork(pool, t.long(), n, r, p), lambda: profk.pages_fork(pool, t, n[:1], r, p),
           lambda: profk.pages_fork(pool, t, n, r[:10].contiguous(), p), lambda: profk.pages_fork(pool, t, n, r, p, grow=-1),
           lambda: profk.pages_fork(None, t, n, r, p), lambda: profk.pages_fork(pool, t, n, r, p, page_size=8), lambda: profk.pages_fork(pool[0], t, n, r, p),
           lambda: profk.pages_fork(pool[..., :12], t, n, r, p), lambda: profk.pages_fork(pool[..., ::2], t, n, r, p), lambda: profk.pages_fork(pool, t[:, :0], n, r, p),
           lambda: profk.pages_fork(pool.cpu(), t, n, r, p), lambda: profk.pages_fork(pool, t.cpu(), n, r, p), lambda: profk.pages_fork(pool[..., 4:20], t, n, r, p),
           lambda: profk.pages_compact(pool, t, r.long()), lambda: profk.pages_compact(pool[:, :, :3], t, r), lambda: profk.pages_compact(pool[..., :7], t, r),
           lambda: profk.pages_copy(pool, p, p[:1]), lambda: profk.pages_copy(pool, p.long(), p.long()),
           lambda: profk.pages_append(k, k, t, n, new[:1], new[:1]), lambda: profk.pages_append(k, k, t, n, new.float(), new.float()),
           lambda: profk.pages_append(k, k, t, n, new[:, :1], new[:, :1]), lambda: profk.pages_append(k, k[:-1], t, n, new, new),
           lambda: profk.pages_append(k, k, t, n, new[..., :4], new[..., :4])]
    bits = _host(pool)
    for i, call in enumerate(bad):
        with pytest.raises(profk.ProfkError):
            call()
            pytest.fail(f"call {i} was not refused")
    torch.cuda.synchronize()
    np.testing.assert_array_equal(_host(pool), bits)


@pytest.mark.parametrize("page,kv_heads,dim", [(1, 1, 8), (8, 1, 96), (16, 2, 64), (16, 8, 128), (64, 4, 64)])
def test_pages_of_every_size_move_whole(page, kv_heads, dim):
    """From one vector per page and layer to thousands: the threads that share a page's copy differ."""
    rng = np.random.default_rng(page * dim)
    pages, live = 300, 140
    refs = np.zeros(pages, dtype=np.int32)
    refs[rng.permutation(pages)[:live]] = 1
    tables = rng.integers(0, pages, (3, 30)).astype(np.int32)
    pool = _pool(3, pages, kv_heads, page, dim, 9)
    before = _host(pool)
    got = profk.pages_compact(pool, _int32(tables), _int32(refs))
    want = oracle.compact(before, tables, refs)
    np.testing.assert_array_equal(got.tables.cpu().numpy(), want[0])
    np.testing.assert_array_equal(_host(pool), before)


@pytest.mark.parametrize("pages", [4096, 4097, 200_000, 700_000])
@pytest.mark.parametrize("held", [0.02, 0.5, 0.98])
def test_compact_plans_in_shares(pages, held):
    rng = np.random.default_rng(pages)
    refs = (rng.random(pages) < held).astype(np.int32) * rng.integers(1, 5, pages).astype(np.int32)
    tables = rng.integers(-1, pages + 1, (7, 500)).astype(np.int32)
    got = profk.pages_compact(None, _int32(tables), _int32(refs))
    want = oracle.compact(np.zeros((1, 2, pages, 1, 1, 1), dtype=np.uint8), tables, refs)
    for g, w in zip(got[:3], want[:3]):
        np.testing.assert_array_equal(g.cpu().numpy(), w)
    assert int(got.live) == want[3]
