"""The error bounds that the header gives for the operators for prompts and drafts, by arithmetic: the steps that an angle and a weight
take, in exact numbers."""
import math
import random
from fractions import Fraction

import numpy as np
import pytest
import torch

INV = 1 / (2 * math.pi)                                  # the constant's 53 bits
TWO_PI = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459")


def _turns_kept(position, frequency):
    """The angle in turns as it is held: the frequency as 64 bits of a turn, the wrapped product's upper 32."""
    turns = frequency * INV
    fraction = min(round(Fraction(turns - round(turns)) * 2 ** 64), 2 ** 63 - 1)
    phase = position * fraction % 2 ** 64
    return Fraction((phase + 2 ** 31) // 2 ** 32, 2 ** 32)


@pytest.mark.parametrize("frequency", [1.0, 7.0, math.pi, 1e5, 0.37, 1e-4, 1e-12, -0.3, 0.5 / INV])
def test_angles(frequency):
    rng = random.Random(1)
    for position in [0, 1, -1, 10 ** 6 + 3, 2 ** 31 - 1, -(2 ** 40)] + [rng.randrange(-(2 ** 40), 2 ** 40) for _ in range(200)]:
        angle = position * Fraction(frequency)
        off = (_turns_kept(position, frequency) - angle / TWO_PI) % 1
        off = min(off, 1 - off) * TWO_PI
        assert off <= abs(angle) / 2 ** 52 + Fraction(abs(position), 2 ** 61) + Fraction(1, 2 ** 30)


@pytest.mark.parametrize("dtype,relative,lift", [(torch.bfloat16, 2.0 ** -8, 0), (torch.float16, 2.0 ** -11, 11)])
def test_weights(dtype, relative, lift):
    """A weight w <= 1 of the row's largest is held as w 2^lift."""
    w = np.concatenate([np.linspace(0.5, 1, 100001), np.exp2(-np.linspace(0, 60, 100001))]).astype(np.float32)
    held = torch.from_numpy(w * np.float32(2 ** lift)).to(dtype).double().numpy() / 2 ** lift
    off = np.abs(held - w.astype(np.float64))
    least = 2.0 ** -36 if dtype == torch.float16 else 0
    assert (off <= np.maximum(relative * w, least)).all()
    assert (off / w)[:100001].max() > 0.9 * relative     # (no smaller power of two would do)
