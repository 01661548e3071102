"""What autograd may and may not expect of the decoding operators: a derivative that they do not have is refused, not left out."""
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


def test_a_second_derivative_is_refused():
    x = torch.randn(3, 50, device="cuda", requires_grad=True)
    loss = profk.logprobs(x, torch.arange(3, device="cuda")).logprob.sum()
    grad, = torch.autograd.grad(loss, x, create_graph=True)
    plain = torch.log_softmax(x, -1)[torch.arange(3), torch.arange(3)].sum()
    assert (grad - torch.autograd.grad(plain, x)[0]).abs().max() < 1e-5
    with pytest.raises(RuntimeError):
        (loss + (grad ** 2).sum()).backward()              # (a penalty on the gradient: its term would count for nothing)
