"""Rotary angles at every frequency and position that the call takes, against exact arithmetic."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def two_pi():
    """2 pi as a fraction, to 2^-200: pi = 16 atan(1/5) - 4 atan(1/239)."""
    one = 1 << 240

    def atan_of_inverse(n):
        total, term, k = 0, one // n, 0
        while term:
            total += (term // (2 * k + 1)) * (-1 if k & 1 else 1)
            term //= n * n
            k += 1
        return total

    return Fraction(2 * (16 * atan_of_inverse(5) - 4 * atan_of_inverse(239)), one)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_angles(dtype):
    """An angle is off by at most 2^-24 of a turn (4e-7 radians), its cosine by 1e-6 more, at frequencies of up to a million radians a position and at the ends
    of the positions' range."""
    from paper_2010_02838_amd import binding as B
    freqs = [1.0, 10.0, 1000.0, 9e5, 999999.999, -1.0, -12345.678, 1e-3, 0.1, 3.14159, 6.283185307179586, 1e-12, 2.0 ** -70, 0.0, -1e-9, 1e-300]
    pos = [0, 1, -1, 2 ** 30, -2 ** 30, 2 ** 31 - 1, -2 ** 31, 1000003, -77777777, 32767, 2 ** 24 + 1]
    turn, half = two_pi(), len(freqs)
    x = torch.randn(len(pos), 2, 2 * half, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(dtype)
    y = torch.empty_like(x)
    B.codistill_rotary(B.rotary_desc(2 * half, (half,), 1.0, dtype, freq=freqs), torch.tensor([pos], dtype=torch.int32, device=DEV), [(x, y)])
    angle = np.array([[float(Fraction(f) * p / turn % 1) * 2 * math.pi for f in freqs] for p in pos])[:, None]
    a, b = np.split(x.double().cpu().numpy(), 2, 2)
    want = np.concatenate([a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)], 2)
    size = np.concatenate([np.hypot(a, b)] * 2, 2)
    err = np.abs(y.double().cpu().numpy() - want)
    assert (err <= 2e-6 * size + (2.0 ** -8 * np.abs(want) if dtype is torch.bfloat16 else 0)).all(), (err / size).max((0, 1))
