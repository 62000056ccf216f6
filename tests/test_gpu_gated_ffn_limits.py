"""The gated feed-forward block where its numbers leave the ordinary range: preactivations near the types' ends, gradients near
the bottom of float16, and more than 2^31 elements in a matrix.  Tolerances as in test_gpu_gated_ffn."""
import pytest
import torch

from paper_2006_07405_b200 import binding as B
from test_gpu_gated_ffn import Block, _check_backward, _check_forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("t", [5, 64])
def test_preactivations_near_the_end_of_the_type_give_no_nan(t, act):
    """a = +-3e30: the activation is a or 0, its slope 1 or 0, and no 0 * inf comes up on the way.  db = dh act(a) <= 1e32 and
    its products with x stay below 1e37, so that every gradient is finite."""
    p = Block(t, 64, 128, torch.bfloat16, scale=100.0)
    p.forward(act)
    p.a.fill_(-3e30)
    p.a[:, ::2] = 3e30
    got = p.backward(act)
    assert all(torch.isfinite(g).all() for g in got.values())
    _check_backward(p, act, got)


@pytest.mark.parametrize("scale", [1e-3, 3e-6])
def test_small_float16_gradients(scale):
    """da and db are held in the type: below 2^-14 their unit is 2^-24 (1e-3 puts some of them there, 3e-6 all)."""
    p = Block(200, 136, 264, torch.float16)
    p.dy.mul_(scale)
    p.forward("silu")
    _check_backward(p, "silu", p.backward("silu"))


@pytest.mark.parametrize("t,d,f", [(1, 1603, 6401), (9, 1603, 6401), (16, 777, 2051), (8, 2048, 4099), (13, 2051, 4096), (2, 4096, 1025)])
def test_few_tokens_with_large_matrices_that_are_not_aligned(t, d, f):
    for pad, skew in ((3, 1), (0, 8)):
        p = Block(t, d, f, torch.bfloat16, pad, skew)
        p.forward("silu")
        _check_forward(p, "silu")
        p.check_edges()


class Rows(Block):
    """Some rows of a block's matrices."""

    def __init__(self, p, rows):
        self.t, self.d, self.f, self.dtype = rows.stop - rows.start, p.d, p.f, p.dtype
        self.wg, self.wu, self.wd = p.wg, p.wu, p.wd
        for name in ("x", "dy", "y", "h", "a", "b"):
            setattr(self, name, getattr(p, name)[rows])


def test_more_than_2_31_elements():
    t, d, f = 131_201, 64, 16_400
    p = Block(t, d, f, torch.bfloat16)
    p.forward("silu")
    got = p.backward("silu")
    cross = (1 << 31) // f
    for lo in (0, cross - 20, t - 40):
        part = Rows(p, slice(lo, lo + 40))
        _check_forward(part, "silu")
        _check_backward(part, "silu", {"dx": got["dx"][lo:lo + 40], "dwg": None, "dwu": None, "dwd": None})
    # weight gradients: the terms' magnitudes by column norms; see test_gpu_gated_ffn for the sums' error
    want = mag = 0.0
    for lo in range(0, t, 8192):
        left, right = p.dy[lo:lo + 8192].double(), p.h[lo:lo + 8192].double()
        want, mag = want + left.T @ right, mag + left.abs().T @ right.abs()
    tol = (t / 16 + 2) * 2.0 ** -22 * mag + 2.0 ** -8 * want.abs()
    assert torch.all((got["dwd"].double() - want).abs() <= tol * (1 + 2.0 ** -8) + 1e-37)


def test_calls_leave_no_status_on_any_stream():
    p = Block(40, 72, 104, torch.float16)
    side = torch.cuda.Stream()
    for stream in (None, side, None):
        p.forward("silu", stream=stream)
        assert B.a2sgd_gated_ffn_status(stream=side) == B.OK and B.a2sgd_gated_ffn_status() == B.OK
