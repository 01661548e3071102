"""Sequences that fill their tables: what has no place is passed over, and no cached token is written over."""
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


@pytest.mark.parametrize("tokens", [1, 3])
def test_children_of_a_full_sequence_leave_the_cache_alone(tokens):
    page, width = 4, 3
    pool = torch.randn(1, 2, 12, 2, page, 16, device="cuda").to(torch.bfloat16)
    tables, lengths = _int32([[0, 1, 2], [3, 4, -1]]), _int32([page * width, 6])
    refs = _int32([1] * 5 + [0] * 7)
    before = pool.clone()
    state = profk.pages_fork(pool, tables, lengths, refs, _int32([0, 0, 1]), grow=tokens, past_room=True)
    assert state.lengths.tolist() == [page * width + tokens] * 2 + [6 + tokens]
    assert int(state.missing) == 2 and state.tables[:2].tolist() == [[0, 1, 2]] * 2
    new = torch.randn(3, tokens, 2, 16, device="cuda").to(pool.dtype)
    k, v = pool[0, 0], pool[0, 1]
    q = torch.randn(3, 4, 16, device="cuda").to(pool.dtype)
    whole = profk.paged_attention(q, k, v, state.tables, _int32([page * width] * 2 + [0]))
    profk.pages_append(k, v, state.tables, state.lengths, new, new)
    held = torch.zeros_like(pool, dtype=torch.bool)          # where the third sequence's tokens went
    for t in range(6, 6 + tokens):
        held[:, :, int(state.tables[2, t // page]), :, t % page] = True
    assert torch.equal(pool[~held], before[~held]) and not torch.equal(pool[held], before[held])
    # other calls take such a length for a full table's
    again = profk.paged_attention(q, k, v, state.tables, state.lengths)
    assert torch.equal(again[0][:2], whole[0][:2])
    on = profk.pages_fork(pool, state.tables, state.lengths, state.refs, _int32([1, 2]), grow=1, past_room=True)
    assert on.lengths.tolist() == [page * width + 1, 7 + tokens]


def test_append_takes_lengths_as_they_are():
    pool = torch.zeros(1, 2, 4, 1, 4, 8, dtype=torch.float16, device="cuda")
    tables = _int32([[0], [1], [2], [3]])
    new = torch.ones(4, 2, 1, 8, dtype=torch.float16, device="cuda")
    profk.pages_append(pool[0, 0], pool[0, 1], tables, _int32([4, 5, 2 ** 31 - 1, -2 ** 31]), new, new)
    want = torch.zeros(4, 4, device="cuda")
    want[0, 2:] = 1                                          # the last two of four tokens
    want[1, 3] = 1                                           # the last token has no place, the one before it has
    for x in range(2):
        assert torch.equal(pool[0, x, :, 0, :, 0].float(), want)


@pytest.mark.parametrize("page", [1, 5, 16])
def test_lengths_past_the_room_against_the_oracle(page):
    rng = np.random.default_rng(page)
    width = 6
    lengths = np.array([0, 1, page * width, page * width - 1, 3 * page, page * width + 100])
    tables = np.arange(6 * width, dtype=np.int32).reshape(6, width)
    refs = np.zeros(200, dtype=np.int32)
    for s, n in enumerate(lengths):
        refs[tables[s, :min(width, -(-n // page))]] = 1
    parents = rng.integers(-1, 6, 20)
    for grow in (0, 1, 7 * page):
        got = profk.pages_fork(None, _int32(tables), _int32(lengths), _int32(refs), _int32(parents), grow=grow, page_size=page, past_room=True)
        want = oracle.fork(np.zeros((1, 2, 200, 1, page, 1)), tables, lengths, refs, parents, grow, past_room=True)
        for g, w in zip(got[:3], want[:3]):
            np.testing.assert_array_equal(g.cpu().numpy(), w)
        assert int(got.missing) == want[3]
