"""Attention where a few tokens outweigh all others by far: the small weights of many tokens together are not small.

Tolerance: that of test_gpu_paged_attention.py for what is relative to sum p |v|, half a unit in the last place of the output
(half its smallest step below that), and for fp16, whose pairs of numbers end at 2^-24 while the largest weight is held at 2^14
or more, 2^-25 / 2^14 = 2^-39 of the largest |v| for each of a sequence's tokens."""
import math

import pytest
import torch

import paper_2608_12573_b200 as profk
from paper_2608_12573_b200 import _build
from test_gpu_paged_attention import _case, _check

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    _build.build()
    profk.lib()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("sink_value", [0.0, 0.5])
def test_a_sink_and_a_long_tail(dtype, dim, sink_value):
    """128 sequences, eight heads, 16384 tokens: the first has score 0, all others of head h lie 2^-d[h] below it (so many
    streams that one warp meets a sink and thousands of tokens of its tail)."""
    seqs, heads, page, width = 128, 8, 32, 512
    d = torch.tensor([10.0, 16.3, 18.0, 20.1, 22.4, 24.4, 25.2, 28.0], device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(dim)
    k, v = (torch.zeros(4, heads, page, dim, dtype=DTYPES[dtype], device="cuda") for _ in range(2))
    k[..., 0] = -d[:, None].to(k.dtype)
    v.copy_(torch.rand(v.shape, generator=g, device="cuda") + 0.5)
    k[0, :, 0], v[0, :, 0] = 0.0, sink_value
    q = torch.zeros(seqs, heads, dim, dtype=k.dtype, device="cuda")
    q[..., 0] = 1.0
    table = torch.cat([torch.zeros(1), torch.arange(width - 1) % 3 + 1]).to(torch.int32).cuda()
    lengths = torch.full((seqs,), width * page, dtype=torch.int32, device="cuda")
    out, lse = profk.paged_attention(q, k, v, table.repeat(seqs, 1), lengths, scale=math.log(2))
    weight = torch.exp2(k[..., 0].double())                                        # (pages, heads, tokens)
    times = torch.bincount(table, minlength=4).double()[:, None, None]
    total = (times * weight).sum((0, 2))
    want = ((times * weight)[..., None] * v.double()).sum((0, 2)) / total[:, None]           # (heads, dim), all terms positive: sum p |v|
    reach = d.double()[:, None] * math.log(2)
    allowed = want * 2 * (reach * 2.0 ** -20 + 2.0 ** -15) + torch.clamp(0.5 * torch.finfo(q.dtype).eps * want, min=2.0 ** -25)
    if dtype == "f16":
        allowed = allowed + width * page * 2.0 ** -39 * 1.5
    assert ((out.double() - want).abs() <= allowed).all()
    want_lse = torch.log(total)
    assert ((lse.double() - want_lse).abs() <= reach[:, 0] * 2.0 ** -20 + 2.0 ** -16 + 2.0 ** -22 * want_lse.abs()).all()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("group", [1, 2, 12])
def test_scores_that_rise_and_fall_far(dtype, group):
    """References that move often, over parts that warps and CTAs join."""
    q, k, v, tables, lengths = _case([900, 901, 3000], 2 * group, 2, 64, 16, dtype, seed=4)
    k *= torch.linspace(0.1, 12, 16, device="cuda").view(1, 1, 16, 1).to(k.dtype)
    _check(q * 2, k, v, tables, lengths, scale=0.3)
