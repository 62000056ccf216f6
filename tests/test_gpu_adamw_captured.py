"""AdamW steps with a gradient scale by value in 8 bits, and norm and step captured in a graph."""
import numpy as np
import pytest
import torch

from paper_2006_07405_b200 import binding as B
from test_gpu_adamw import F32, HYPER, Problem, _step8

pytestmark = pytest.mark.gpu


def test_8_bit_step_with_a_scale_is_defined_to_the_bit():
    numel = [5, 3000, 70_001]
    p = Problem(numel, torch.bfloat16, 0, 8, torch.bfloat16, seed=21)
    scale = torch.tensor([0.37], device="cuda")
    live = p.flat([torch.ones(n) for n in numel]) > 0
    for step in (1, 2, 77):
        w, g = p.flat(p.w).astype(F32), p.flat(p.g).astype(F32) * F32(0.37)
        state = [t.cpu().numpy() for t in (p.m, p.v, p.ms, p.vs)]
        B.a2sgd_adamw_step(p.plan, step=step, grad_scale=scale, **HYPER)
        ref = _step8(w, g, *state, step, **HYPER)
        assert np.array_equal(p.flat(p.w).astype(F32)[live], ref[0][live])
        for got, want in zip((p.m, p.v, p.ms, p.vs), ref[1:]):
            assert np.array_equal(got.cpu().numpy().astype(F32), want)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_step_replays_its_own_step_number(bits):
    """Norm and step in a graph: every replay is the eager call with the step number of the capture."""
    p, q = Problem([70_001, 300], bits=bits, seed=2), Problem([70_001, 300], bits=bits, seed=2)
    out, ref = torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.a2sgd_adamw_grad_norm(p.plan, 0.5, out)
        B.a2sgd_adamw_step(p.plan, step=9, grad_scale=out[1:], **HYPER)
    for _ in range(3):
        graph.replay()
        B.a2sgd_adamw_grad_norm(q.plan, 0.5, ref)
        B.a2sgd_adamw_step(q.plan, step=9, grad_scale=ref[1:], **HYPER)
    torch.cuda.synchronize()
    for a, b in zip([t for t in (p.wbuf, p.m, p.v, p.ms, p.vs, out) if t is not None],
                    [t for t in (q.wbuf, q.m, q.v, q.ms, q.vs, ref) if t is not None]):
        assert torch.equal(a, b)
