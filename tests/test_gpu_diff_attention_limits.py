"""Differential attention where its numbers or layouts are at their limits, against the formula in float64 (tolerances as in
test_gpu_diff_attention.py)."""
import math

import numpy as np
import pytest
import torch

from test_gpu_diff_attention import BF, DEV, F32, TOL, Problem, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale", [0.0, 1e-12, 1e-20])
def test_lambdas_near_zero_and_small_scales(dtype, scale):
    """A lambda of zero, below the normal numbers or close above them: its logarithm, and what that is over the scale, stay finite, and the other rows'
    gradients are what they were.  (Small scales: all weights are alike.  dq and dk without the floor that `check` gives them.)"""
    p = Problem(dtype, [40, 70], [40, 70], 4, 2, 64, True, True, seed=11, scale=scale)
    for i, lam in enumerate((0.0, 1e-40, -1e-40, 1e-30, -1e-30, -0.0)):
        p.lam[:, i::7] = lam
    p.want()
    p.run()
    p.check()
    for name, at, keys in (("dq", 1, False), ("dk", 2, True)):
        got = torch.cat([p.rows(getattr(p, name), b, keys).flatten() for b in range(2)])
        close(got, np.concatenate([p.ref[b][at].ravel() for b in range(2)]), TOL[dtype] * (8 if dtype is F32 else 1), name)
