"""Layer norm forward and backward captured in a graph: every replay gives the eager calls' bits."""
import pytest
import torch

from paper_2006_07405_b200 import binding as B
from test_gpu_layer_norm import _problem, _statistics

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,d,dtype", [(300, 1600, torch.bfloat16), (37, 1001, torch.float32), (5, 8200, torch.float16)])
def test_calls_can_be_captured_in_a_graph(rows, d, dtype):
    x, dy, w, b = _problem(rows, d, dtype, torch.float32)
    mean, rstd = _statistics(x)
    work = torch.empty(B.a2sgd_layer_norm_workspace(rows, d), dtype=torch.uint8, device="cuda")
    outs = [[torch.empty_like(x), torch.empty_like(mean), torch.empty_like(mean), torch.empty_like(x), torch.empty_like(w),
             torch.empty_like(w)] for _ in range(2)]

    def calls(y, m, r, dx, dw, db):
        B.a2sgd_layer_norm_forward(x, w, b, y, m, r)
        B.a2sgd_layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db, work)

    calls(*outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(*outs[1])
    for _ in range(2):
        for t in outs[1]:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(outs[1], outs[0]):
            assert torch.equal(got, want)
