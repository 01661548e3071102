"""The decoding operators together: a beam search over a paged cache against the same model without one."""
import importlib.util
import os

import pytest
import torch

import paper_2608_12573_b200 as profk
from paper_2608_12573_b200 import _build

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    _build.build()
    profk.lib()
    spec = importlib.util.spec_from_file_location("beam_search", os.path.join(ROOT, "examples", "beam_search.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("searches,beams,steps,page", [(1, 1, 5, 16), (3, 4, 20, 16), (2, 7, 33, 8), (5, 3, 18, 5)])
def test_beam_search(example, searches, beams, steps, page):
    model = example.Decoder(1009, seed=searches)
    first = torch.arange(searches, device="cuda") * 3 + 1
    with torch.no_grad():
        sequences, scores, refs, tables, lengths = example.beam_search(model, first, beams, steps, page_size=page, check=True)
        again = model.dense_scores(sequences.flatten(0, 1)).view(searches, beams)
    # Activations are rounded to bf16 five times a layer and token (2^-9 relative each) and the logits once: a step's log
    # probability may be off by a few times 2^-8 of logits of some units, 0.1 at worst, and a sequence's by `steps` of them.
    assert (scores.double() - again).abs().max() < 0.1 * steps
    assert (scores[:, :-1] >= scores[:, 1:]).all()
    assert (sequences[:, :, 0] == first[:, None]).all()
    for s in range(searches):
        assert len({tuple(x) for x in sequences[s].tolist()}) == beams      # no continuation twice
    # the cache's counts are those of the tables' entries
    assert (lengths == steps + 1).all()
    held = -(-(steps + 1) // page)
    assert (tables[:, :held] >= 0).all()
    counts = torch.bincount(tables[:, :held].flatten(), minlength=refs.shape[0])
    assert torch.equal(counts.int(), refs)


def test_the_first_step_is_the_exact_one(example):
    """One step from one token: the beams are the best tokens of the model's distribution."""
    model = example.Decoder(4001, seed=9)
    first = torch.tensor([7, 8], device="cuda")
    with torch.no_grad():
        sequences, scores, *_ = example.beam_search(model, first, 6, 1)
        logits = model.step(first, torch.zeros(2, 2, 2, 2, 16, 64, dtype=torch.bfloat16, device="cuda"),
                            torch.arange(2, dtype=torch.int32, device="cuda")[:, None], torch.ones(2, dtype=torch.int32, device="cuda"))
    want = profk.topk(logits, 6)[1]
    assert torch.equal(sequences[:, :, 1], want)
    logp = torch.log_softmax(logits.double(), -1).gather(1, want)
    assert (scores.double() - logp).abs().max() < 1e-4
