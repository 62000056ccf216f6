"""The training operators with every matrix or tensor in a layout of its own: some aligned, some not, rows of different strides.
Tolerances as in the operators' own tests; nothing outside of the rows is written."""
import random

import pytest
import torch

from paper_2006_07405_b200 import binding as B
import test_gpu_adamw as A
import test_gpu_gated_ffn as G
import test_gpu_layer_norm as L

pytestmark = pytest.mark.gpu
LAYOUTS = [(0, 0), (8, 0), (0, 8), (16, 16), (1, 0), (0, 1), (3, 5), (8, 1), (5, 8)]     # elements between rows, before the first


class Mixed(G.Block):
    """A block whose matrices draw their layouts one by one."""

    def __init__(self, t, d, f, dtype, seed):
        self.layouts, self.rng = {}, random.Random(seed)
        super().__init__(t, d, f, dtype, seed=seed)

    def rows(self, name, values):
        r, c = values.shape
        pad, skew = self.layouts[name] = self.rng.choice(LAYOUTS)
        buf = torch.full((r * (c + pad) + skew + 64,), 9.0, device="cuda").to(self.dtype)
        out = buf[skew:skew + r * (c + pad)].view(r, c + pad)[:, :c]
        out.copy_(values)
        self.bufs[name] = (buf, r, c)
        return out

    def check_edges(self):
        for name, (buf, r, c) in self.bufs.items():
            pad, skew = self.layouts[name]
            end = skew + r * (c + pad)
            assert torch.all(buf[:skew] == 9.0) and torch.all(buf[end:] == 9.0), name
            assert torch.all(buf[skew:end].view(r, c + pad)[:, c:] == 9.0), name


SIZES = [(1, 1, 1), (2, 1, 3), (1, 64, 128), (3, 8, 8), (16, 24, 40), (16, 1600, 640), (17, 8, 7), (18, 7, 8), (40, 64, 63), (64, 72, 1),
         (33, 1, 65), (256, 64, 64), (257, 129, 136), (130, 264, 520), (300, 520, 136), (90, 1024, 1001), (700, 80, 72)]


@pytest.mark.parametrize("t,d,f", SIZES)
@pytest.mark.parametrize("seed", range(4))
def test_gated_block(t, d, f, seed):
    dtype, act = ((torch.bfloat16, "silu"), (torch.float16, "gelu_tanh"))[seed % 2]
    p = Mixed(t, d, f, dtype, 1000 * seed + t + d + f)
    p.forward(act)
    G._check_forward(p, act)
    G._check_backward(p, act, p.backward(act))
    p.check_edges()


@pytest.mark.parametrize("rows,d", [(1, 1), (1, 24), (5, 8), (70, 64), (33, 257), (9, 1001), (300, 1600), (20000, 40), (2500, 777), (3, 8200)])
@pytest.mark.parametrize("seed", range(4))
def test_layer_norm(rows, d, seed):
    rng = random.Random(seed * 100 + rows + d)
    dtype, param = L.TYPES[(seed + rows) % len(L.TYPES)]
    x0, dy0, w, b = L._problem(rows, d, dtype, param, seed=seed)
    bufs = []

    def lay(values):
        pad, skew = rng.choice(LAYOUTS)
        out, buf = L._rows(values, dtype, pad, skew)
        bufs.append((buf, pad, skew))
        return out

    x, dy, y, dx = lay(x0), lay(dy0), lay(torch.zeros_like(x0)), lay(torch.zeros_like(x0))
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.a2sgd_layer_norm_forward(x, w, b, y, mean, rstd, 1e-5)
    L._check_forward(x, w, b, y, mean, rstd, 1e-5)
    mean, rstd = L._statistics(x)
    # the parameters' gradients at odd addresses
    dw, db = (torch.full((d + 3,), 5.0, device="cuda").to(param) for _ in range(2))
    work = torch.empty(B.a2sgd_layer_norm_workspace(rows, d), dtype=torch.uint8, device="cuda")
    B.a2sgd_layer_norm_backward(dy, x, w, mean, rstd, dx, dw[1:d + 1], db[2:d + 2], work)
    L._check_backward(dy, x, w, mean, rstd, dx, dw[1:d + 1], db[2:d + 2])
    assert dw[0] == 5 and torch.all(dw[d + 1:] == 5) and torch.all(db[:2] == 5) and db[d + 2] == 5
    for buf, pad, skew in bufs:
        assert torch.all(buf[:skew] == 9.0) and torch.all(buf[skew:].view(rows, d + pad)[:, d:] == 9.0)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gtype,copy", [(torch.float32, None), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.bfloat16)])
def test_adamw(bits, gtype, copy):
    """The same list with every tensor's weights, gradients and copy at other addresses: the same bits as all aligned."""
    numel = [1, 7, 256, 300, 2048, 5000, 70_001, 4096]
    p = A.Problem(numel, gtype, 0, bits, copy, seed=3)
    rng = random.Random(5)

    def moved(tensors):
        out = []
        for t in tensors:
            skew = rng.choice([0, 1, 2, 4, 8])
            buf = torch.full((t.numel() + skew + 16,), 3.0, dtype=t.dtype, device="cuda")
            buf[skew:skew + t.numel()] = t
            out.append((buf, skew, buf[skew:skew + t.numel()]))
        return out

    w, g, c = moved(p.w), moved(p.g), moved(p.c) if copy else None
    state = [t.clone() if t is not None else None for t in (p.m, p.v, p.ms, p.vs)]
    plan = B.a2sgd_adamw_create([t[2] for t in w], [t[2] for t in g], *state, [t[2] for t in c] if copy else None)
    out, ref = torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda")
    for step in (1, 2, 3):
        B.a2sgd_adamw_grad_norm(p.plan, 0.5, ref)
        B.a2sgd_adamw_grad_norm(plan, 0.5, out)
        assert torch.all((out - ref).abs() <= 2 * A.U * ref.abs())          # the squares' sum in another order
        B.a2sgd_adamw_step(p.plan, step=step, grad_scale=ref[1:], **A.HYPER)
        B.a2sgd_adamw_step(plan, step=step, grad_scale=ref[1:], **A.HYPER)
    for a, b in zip(state, (p.m, p.v, p.ms, p.vs)):
        assert a is None or torch.equal(a, b)
    for moved_list, tensors in ((w, p.w), (c, p.c)):
        for (buf, skew, t), same in zip(moved_list or [], tensors):
            assert torch.equal(t, same)
            assert torch.all(buf[:skew] == 3.0) and torch.all(buf[skew + t.numel():] == 3.0)
