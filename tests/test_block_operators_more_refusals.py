"""More of what the attention's and the residual connection's entry points refuse, through the C ABI, before anything is launched: no GPU is needed."""
import math

import pytest

from paper_2006_07405_b200 import binding as B
from test_block_operators_refusals import FAKE, at, heads, residual, rows, shape


def backward(s, dout=None, q=None, k=None, v=None, o=None, dq=None, dk=None, dv=None):
    t = heads()
    first, rest = [dout or t, q or t, k or t, v or t, o or t], [dq, dk, dv]
    return B.lib().a2sgd_window_attention_backward(at(s), *(at(x) for x in first), FAKE, *(at(x) for x in rest), FAKE, 1 << 30, 0, None)


def test_packed_queries_with_gradients_or_outputs_that_are_not():
    packed, s = heads(seq=0), shape(q_ranges=FAKE)
    assert backward(s, q=packed, dq=packed, o=packed) == B.ERR_ARG                      # dout has a plane for each sequence
    assert backward(s, q=packed, dq=packed, dout=packed) == B.ERR_ARG                   # o has
    assert backward(s, q=packed, dk=heads(), o=packed) == B.ERR_ARG


@pytest.mark.parametrize("scale", [1e-46, 5e-324, 2.5e38, 3.5e38, 1e308])
def test_scales_that_fp32_does_not_hold(scale):
    """In fp32, and times log2 e in fp32, a scale is neither 0 nor infinite."""
    t, s = heads(), shape(scale=scale)
    assert B.lib().a2sgd_window_attention_forward(at(s), at(t), at(t), at(t), at(t), None, None, 0, 0, None) == B.ERR_ARG
    assert backward(s, dq=t, dk=t, dv=t) == B.ERR_ARG


@pytest.mark.parametrize("bad", [dict(alpha=1e39), dict(alpha=-1e300), dict(eps=1e39), dict(alpha=math.inf)])
def test_factors_that_fp32_does_not_hold(bad):
    r, s = rows(), residual(pre_rstd=FAKE, **bad)
    assert B.lib().a2sgd_residual_norm_forward(at(s), at(r), at(r), at(r), at(r), 0, None) == B.ERR_ARG
    if "alpha" in bad:      # eps is not read by the backward pass
        assert B.lib().a2sgd_residual_norm_backward(at(s), at(r), at(r), at(r), at(r), at(r), at(r), None, FAKE, 1 << 30, 0, None) == B.ERR_ARG
