"""The rotation has a derivative in what is turned and in nothing else: frequencies that require one are refused, whether or not x
requires one, too.  On the CPU with a stand-in for the native call, and on a GPU."""
import pytest
import torch

import paper_2608_12573_b200 as profk
from paper_2608_12573_b200 import _build, decode


class _StandIn:
    """Doubles x."""
    calls = 0

    def rotary(self, x, positions, frequencies, interleaved, magnitude, inverse):
        self.calls += 1
        return x * 2


@pytest.fixture
def native(monkeypatch):
    stand_in = _StandIn()
    monkeypatch.setattr(decode, "_native", stand_in)
    return stand_in


def _arguments(device="cpu"):
    x = torch.ones(3, 2, 4, device=device)
    return x, torch.arange(3, device=device), torch.ones(2, dtype=torch.float64, device=device)


def test_frequencies_that_require_a_gradient_beside_an_x_that_does(native):
    x, at, f = _arguments()
    x.requires_grad_(True)
    with pytest.raises(profk.ProfkError, match="frequencies requires a gradient"):
        profk.rotary(x, at, f.clone().requires_grad_(True))
    with pytest.raises(profk.ProfkError, match="frequencies requires a gradient"):
        profk.rotary(x * 1, at, f.clone().requires_grad_(True) * 2)          # neither is a leaf
    assert native.calls == 0


def test_what_is_not_refused(native):
    x, at, f = _arguments()
    x.requires_grad_(True)
    grad, = torch.autograd.grad(profk.rotary(x, at, f).sum(), x, create_graph=True)
    assert torch.equal(grad, torch.full_like(x, 2.0))
    with torch.no_grad():
        assert not profk.rotary(x, at, f.clone().requires_grad_(True)).requires_grad
    assert profk.rotary(x, at, f.clone().requires_grad_(True).detach()).requires_grad


@pytest.mark.gpu
@pytest.mark.parametrize("trained", [False, True])
def test_on_a_gpu(trained):
    _build.build()
    x, at, f = _arguments("cuda")
    x.requires_grad_(trained)
    with pytest.raises(profk.ProfkError, match="requires a gradient"):
        profk.rotary(x, at, f.clone().requires_grad_(True))
    assert profk.rotary(x, at, f).requires_grad == trained
