"""The waits inside the attention of a chunk are bounded.  Here they run out (no poll is granted, so that a wait gives up when what it
waits for has not come yet; nothing hangs and nothing faults): every output is NaN, and the next call is as if nothing had been."""
import ctypes

import numpy as np
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


def _case(lengths, news, heads, kv_heads, dim, page, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda")
    g.manual_seed(dim + page)
    width = -(-max(lengths) // page)
    tables = torch.arange(len(lengths) * width, dtype=torch.int32, device="cuda").view(len(lengths), width)
    k, v = (torch.randn(tables.numel(), kv_heads, page, dim, generator=g, device="cuda").to(dtype) for _ in range(2))
    q = torch.randn(sum(news), heads, dim, generator=g, device="cuda").to(dtype)
    starts = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32, device="cuda")
    return q, k, v, tables, torch.tensor(lengths, dtype=torch.int32, device="cuda"), starts


def _call(case):
    return profk.paged_attention_chunk(*case[:5], starts=case[5])


# page 16: copied by tile; 7: token by token.  heads 10 on 2: queries row by row.  The second case is longer than the ring of stages.
@pytest.mark.parametrize("page", [16, 7])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads", [(4, 2), (10, 2)])
@pytest.mark.parametrize("lengths,news", [([300, 40], [200, 40]), ([9000, 8000, 9500], [300, 2, 260])])
def test_waits_that_run_out_leave_no_numbers_and_the_next_call_is_right(page, dim, heads, kv_heads, lengths, news):
    case = _case(lengths, news, heads, kv_heads, dim, page)
    want = _call(case)
    torch.cuda.synchronize()
    polls = profk.lib().profk_debug_set_chunk_wait_polls
    try:
        assert polls(ctypes.c_int64(0)) == 0
        got = _call(case)
        torch.cuda.synchronize()
    finally:
        polls(ctypes.c_int64(-1))
    assert torch.isnan(got[0]).all() and torch.isnan(got[1]).all()
    for _ in range(2):
        again = _call(case)
        torch.cuda.synchronize()
        assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])
