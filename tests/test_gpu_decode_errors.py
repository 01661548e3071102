"""The exceptions of the decoding operators' binding."""
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


def test_memory_that_is_not_to_be_had_raises_what_torch_raises():
    """New tables of 2^20 sequences by 65536 pages would be 275 GB."""
    tables = torch.zeros(1, 65536, dtype=torch.int32, device="cuda")
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    parents = torch.zeros(1 << 20, dtype=torch.int32, device="cuda")
    with pytest.raises(torch.OutOfMemoryError):
        profk.pages_fork(None, tables, one, one, parents, page_size=16)
    got = profk.pages_fork(None, tables, one, one, parents[:3], page_size=16)          # and goes on
    assert got.lengths.tolist() == [1, 1, 1]
