"""AdamW at the ends of its arguments.  Tolerances as in test_gpu_adamw."""
import numpy as np
import pytest
import torch

from paper_2006_07405_b200 import binding as B
from test_gpu_adamw import F32, HYPER, Problem, _formula

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [dict(eps=1e39), dict(eps=1e300), dict(lr=1e39), dict(lr=1e30, weight_decay=1e30),
                                 dict(lr=3e38, beta1=0.9999)])
def test_coefficients_beyond_fp32_are_refused(bits, bad):
    p = Problem([300], bits=bits)
    before = [t.clone() for t in (p.wbuf, p.m, p.v)]
    with pytest.raises(B.A2SGDError) as e:
        B.a2sgd_adamw_step(p.plan, step=1, **{**HYPER, **bad})
    assert e.value.status == B.ERR_ARG
    for a, b in zip((p.wbuf, p.m, p.v), before):
        assert torch.equal(a, b)


@pytest.mark.parametrize("eps", [1e-8, 1.0, 2.0 ** 59, 2.0 ** 61, 2.0 ** 100, 1e38, 3e38])
@pytest.mark.parametrize("gscale", [1e-2, 1e10])
def test_large_eps(eps, gscale):
    """The update is m / eps then, tiny but right; weights of zero show it."""
    p = Problem([5000], gscale=gscale)
    p.w[0].zero_()
    w, g, m, v = p.flat(p.w), p.flat(p.g), p.m.double().cpu().numpy(), p.v.double().cpu().numpy()
    h = {**HYPER, "eps": float(F32(eps))}
    B.a2sgd_adamw_step(p.plan, step=3, **h)
    for (ref, tol), got in zip(_formula(w, g, m, v, 3, **h), (p.flat(p.w), p.m.double().cpu().numpy(), p.v.double().cpu().numpy())):
        assert np.all(np.abs(got - ref) <= tol)
