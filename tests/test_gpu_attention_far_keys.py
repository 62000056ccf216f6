"""float16: many keys of little weight beside a first one of nearly all."""
import math

import pytest
import torch

from paper_2006_07405_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lq", [1, 2, 140])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gap", [14.0, 17.5, 18.5])
def test_their_sum_is_in_the_output(lq, d, gap):
    """Scores of 0 beside one of `gap`, values of 1 beside one of 0: the output is n e^-gap / (1 + n e^-gap) of n far keys.

    P is held as float16 about a reference that leaves the row's largest one at 2^6 at least: a P below float16's normal numbers is off by 2^-25 of 2^6,
    2^-31, which n far keys may all be in the same direction; others by half a step, 2^-11.  exp in fp32: 2^-21 (2 + gap); sums of n terms: n 2^-24;
    the output's own half step.
    """
    n = 20000
    q, k = torch.zeros((1, lq, 2, d), dtype=torch.float16, device="cuda"), torch.zeros((1, n, 2, d), dtype=torch.float16, device="cuda")
    v, o = torch.ones_like(k), torch.empty_like(q)
    q[..., 0], k[:, 0, :, 0], v[:, 0] = 1.0, gap, 0.0
    work = torch.empty(B.a2sgd_window_attention_workspace(q, k, None, 0, 1), dtype=torch.uint8, device="cuda")
    lse = torch.empty((1, 2, lq), device="cuda")
    B.a2sgd_window_attention_forward(q, k, v, o, lse, scale=1.0, workspace=work)
    far = torch.arange(n - lq, n, device="cuda", dtype=torch.float64) * math.exp(-gap)
    want = (far / (1.0 + far))[None, :, None, None].expand_as(o)
    bound = n * 2.0 ** -31 + want * (2 * 2.0 ** -11 + 2.0 ** -21 * (2 + gap) + n * 2.0 ** -24) + 2.0 ** -25
    assert ((o.double() - want).abs() <= bound).all(), (o.double() - want).abs().max().item()
    assert ((lse.double() - (gap + torch.log1p(far))).abs() <= n * 2.0 ** -24 + 2.0 ** -21 * (2 + 2 * gap)).all()


@pytest.mark.parametrize("lq", [2, 300])
def test_scores_that_rise_again_and_again(lq):
    """Every key's score is the highest so far, by steps from a fraction of a bit to many: no probability leaves float16's range."""
    for step in (0.01, 0.05, 0.3, 1.0, 7.0):
        n, d = 700, 64
        q, k = torch.zeros((1, lq, 1, d), dtype=torch.float16, device="cuda"), torch.zeros((1, n, 1, d), dtype=torch.float16, device="cuda")
        gen = torch.Generator("cuda").manual_seed(1)
        v, o = torch.empty((1, n, 1, d), device="cuda").normal_(generator=gen).half(), torch.empty_like(q)
        q[..., 0], k[0, :, 0, 0] = 1.0, (torch.arange(n, device="cuda") * step).half()
        work = torch.empty(B.a2sgd_window_attention_workspace(q, k, None, 0, 1), dtype=torch.uint8, device="cuda")
        B.a2sgd_window_attention_forward(q, k, v, o, scale=1.0, workspace=work)
        i, j = torch.arange(n - lq, n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
        x = k[0, :, 0, 0].double()[None].expand(lq, n).masked_fill(j > i, -math.inf)
        p = torch.softmax(x, 1)
        want = p @ v[0, :, 0].double()
        # half a step of P and of the output; exp of a score up to 4893 in fp32: 2^-21 (2 + score); P below the normal numbers; fp32 sums
        size = p @ v[0, :, 0].double().abs()
        bound = size * (2.0 ** -11 + 2 * 2.0 ** -21 * (2 + x.amax().item()) + n * 2.0 ** -24) + want.abs() * 2.0 ** -11 + 2.0 ** -31 * v[0, :, 0].double().abs().sum(0) + 2.0 ** -25
        assert ((o[0, :, 0].double() - want).abs() <= bound).all(), step
