"""What the operators of a differential-attention layer refuse at the limits of their numbers and layouts, and what they do not, without a GPU: every call
below ends in the checks in front of any launch."""
import ctypes

import pytest
import torch

from paper_2010_02838_amd import binding as B
from test_operators_host import BAD, UNSUPPORTED, at, attn, backward, forward


def test_scales_of_the_gradients():
    for scale, rc in ((2.0 ** -101, UNSUPPORTED), (1e-45, UNSUPPORTED), (2.0 ** -100, B.CD_ERR_WORKSPACE_TOO_SMALL), (0.0, B.CD_ERR_WORKSPACE_TOO_SMALL)):
        assert backward(attn(scale=scale), room=0) == rc, scale
