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


@pytest.mark.parametrize("kw", [dict(tq=0), dict(tk=0), dict(tq=0, tk=0)])
def test_packed_rows_need_the_longest_sequence(kw):
    """(A longest sequence of none would leave every row unwritten.)  Without rows there is nothing to say."""
    packed = dict(q_starts=4096, k_starts=4096, q_rows=20, k_rows=24)
    assert forward(attn(**dict(packed, **kw))) == BAD and b"longest" in B.lib.codistill_last_error()
    assert backward(attn(**dict(packed, **kw))) == BAD
    assert B.lib.codistill_diff_attention_workspace_bytes(ctypes.byref(attn(**dict(packed, **kw))), 0, ctypes.byref(ctypes.c_size_t())) == BAD
    none = dict(packed, q_rows=0 if "tq" in kw else 20, k_rows=0 if "tk" in kw else 24)
    assert B.lib.codistill_diff_attention_workspace_bytes(ctypes.byref(attn(**dict(none, **kw))), 0, ctypes.byref(ctypes.c_size_t())) == B.CD_OK
