"""The operators for prompts and drafts where their counters change or their plans are longest: histories around the length from which
counters have 32 bits, and prompts of many blocks of rows to one key-value head."""
import pytest
import torch

import paper_2608_12573_b200 as profk
from paper_2608_12573_b200 import _build
from test_gpu_adjust_logits import _bits, _check as _check_logits, _logits
from test_gpu_paged_attention_chunk import _case, _check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    _build.build()
    profk.lib()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("history", [32766, 32767, 32768, 32769, 65537])
@pytest.mark.parametrize("vocab", [2, 5000, 70000])
def test_one_token_in_all_places_of_a_history(history, vocab):
    """Counters of 16 bits hold 15 of a count and one for the prompt; a neighbour's must not feel either."""
    x = _logits(4, vocab)
    tokens = torch.full((4, history), vocab - 2, device="cuda")
    tokens[3, 1::2] = vocab - 1                                  # the two share a word
    prompts = torch.tensor([0, 1, history, history // 2], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([history, history, history, history - 1], dtype=torch.int32, device="cuda")
    got = _check_logits(x, tokens, lengths, prompts, repetition=1.5, frequency=2.0 ** -10, presence=0.25)
    assert torch.equal(_bits(got[:, :vocab - 2]), _bits(x[:, :vocab - 2]))
    assert torch.equal(_bits(got[:3, vocab - 1]), _bits(x[:3, vocab - 1]))


@pytest.mark.parametrize("heads,kv_heads,dim,news,lengths", [(64, 1, 64, [1500, 3], [1500, 800]), (48, 1, 128, [1100], [1333]), (130, 2, 256, [300, 0, 200], [300, 9, 777])])
def test_many_blocks_of_rows_to_a_key_value_head(heads, kv_heads, dim, news, lengths):
    q, k, v, tables, lengths, starts = _case(lengths, news, heads, kv_heads, dim, 16, "bf16", seed=heads)
    out, lse = profk.paged_attention_chunk(q, k, v, tables, lengths, starts=starts)
    again = profk.paged_attention_chunk(q, k, v, tables, lengths, starts=starts)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    group = heads // kv_heads
    some = [0, group // 2 + 1, group - 1]                        # (the oracle's time: a few of the first key-value head's)
    _check(q[:, some], k[:, :1], v[:, :1], tables, lengths, starts, result=(out[:, some], lse[:, some]))
    some = [(kv_heads - 1) * group, heads - 2]                   # ... and of the last one's
    _check(q[:, some], k[:, -1:], v[:, -1:], tables, lengths, starts, result=(out[:, some], lse[:, some]))
