"""Log probabilities and their gradient where sizes, values and buffers reach the limits of what is accepted."""
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


def test_as_many_rows_as_are_accepted():
    """2^31 - 1 rows of one logit: a row's number and the step to the next one together pass 31 bits.  Of one logit the
    log-sum-exp is the logit itself, exactly."""
    rows = 2 ** 31 - 1
    x = torch.empty(rows, 1, dtype=torch.float16, device="cuda")
    step = 1 << 27
    for r in range(0, rows, step):
        n = min(step, rows - r)
        x[r:r + n, 0] = ((torch.arange(r, r + n, device="cuda") * 7919) % 4096 - 2048).half()
    lse = profk.logprobs(x, entropy=False).lse
    for r in range(0, rows, step):
        assert torch.equal(lse[r:r + step], x[r:r + step, 0].float())
