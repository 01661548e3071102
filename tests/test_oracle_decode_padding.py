"""The oracle's gradient where the list of alternatives has places without a token."""
import numpy as np
import pytest

from oracle import decode as oracle


@pytest.mark.parametrize("top,token", [([2, -1, 3], 3), ([-1, -1], -1), ([9, 0, 100], 9)])
def test_gradient_with_places_without_a_token_against_differences(top, token):
    rng = np.random.default_rng(3)
    x, h = rng.normal(size=9) * 2, 1e-6
    args = (0.8, token, 0.7, -0.4, 1.3, np.array(top), rng.normal(size=len(top)))
    grad, _ = oracle.logprobs_gradient_row(x, *args)
    for v in range(9):
        a, b = x.copy(), x.copy()
        a[v] += h
        b[v] -= h
        assert grad[v] == pytest.approx((oracle.logprobs_loss(a, *args) - oracle.logprobs_loss(b, *args)) / (2 * h), abs=1e-6)
