"""Queries that are not numbers, and keys: what sees them is not a number, by the kernel for few queries as by the one for many."""
import math

import pytest
import torch

from paper_2006_07405_b200 import binding as B

pytestmark = pytest.mark.gpu


def normal(gen, *shape):
    return torch.empty(shape, device="cuda").normal_(generator=gen).to(torch.bfloat16)


@pytest.mark.parametrize("keys, d", [(100, 64), (3000, 64), (20000, 64), (9000, 128)])
@pytest.mark.parametrize("room", [True, False])
def test_a_query_that_is_not_a_number_over_caches_of_all_lengths(keys, d, room):
    """Shares of one CTA, of a cluster, and of a second launch; as in the same query among many."""
    gen = torch.Generator("cuda").manual_seed(keys)
    q, k, v = normal(gen, 1, 2, 2, d), *(normal(gen, 1, keys, 1, d) for _ in range(2))
    q[0, 1, 0, 5] = math.nan
    work = torch.empty(B.a2sgd_window_attention_workspace(q, k, None, 0, 1, aligned=True), dtype=torch.uint8, device="cuda") if room else None
    o, lse = torch.zeros_like(q), torch.zeros((1, 2, 2), device="cuda")
    B.a2sgd_window_attention_forward(q, k, v, o, lse, workspace=work)
    assert torch.isnan(o[0, 1, 0]).all() and torch.isnan(lse[0, 0, 1])
    assert torch.isfinite(o[0, 0]).all() and torch.isfinite(o[0, 1, 1]).all() and torch.isfinite(lse[0, :, 0]).all() and torch.isfinite(lse[0, 1, 1])
    # a run of keys that are none, in one warp's share of many
    q = normal(gen, 1, 2, 2, d)
    k[0, keys // 2 - 20:keys // 2 + 20] = math.nan
    B.a2sgd_window_attention_forward(q, k, v, o, lse, workspace=work)
    assert torch.isnan(o).all() and torch.isnan(lse).all()


def test_a_query_that_sees_only_scores_of_minus_infinity():
    """Not one that sees nothing: the softmax of such scores is not a number, by either kernel."""
    for lq in (2, 200):
        q, k = torch.ones((1, lq, 1, 64), dtype=torch.bfloat16, device="cuda"), -torch.ones((1, 150, 1, 64), dtype=torch.bfloat16, device="cuda")
        q[0, -1] = math.inf
        o, lse = torch.zeros_like(q), torch.zeros((1, 1, lq), device="cuda")
        work = torch.empty(B.a2sgd_window_attention_workspace(q, k, 40, 1, 1), dtype=torch.uint8, device="cuda")
        B.a2sgd_window_attention_forward(q, k, k, o, lse, window=40, sinks=1, workspace=work)
        assert torch.isnan(o[0, -1]).all() and torch.isnan(lse[0, 0, -1]) and torch.isfinite(o[0, :-1]).all()
        empty = max(0, lq - 150)
        assert torch.isneginf(lse[0, 0, :empty]).all() and torch.isfinite(lse[0, 0, empty:-1]).all() and not o[0, :empty].any()
