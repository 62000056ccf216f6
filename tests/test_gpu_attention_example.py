"""The operators of a transformer block as they are used together: the example runs, and its gradients are the network's."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("train_attention_block", os.path.join(ROOT, "examples", "train_attention_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _definition(net, x, p):
    """The network in 64 bits from torch's own operations, for autograd."""
    h, kv, n, eps = net.heads, net.kv_heads, net.head_dim, 1e-5
    rms = lambda a, w: a * (a.square().mean(1, keepdim=True) + eps).rsqrt() * w  # noqa: E731

    def turned(a):
        pairs, out = n // 2, a.clone()
        for j in range(pairs):
            axis, l = divmod(j, n // 4)
            angle = (net.positions[axis].double() * 10000.0 ** -(l / (n // 4)))[:, None]
            u, v = a[..., j], a[..., j + pairs]
            out[..., j], out[..., j + pairs] = u * angle.cos() - v * angle.sin(), u * angle.sin() + v * angle.cos()
        return out

    i, j = torch.arange(net.rows, device=x.device)[:, None], torch.arange(net.rows, device=x.device)[None]
    hidden = ~((j <= i) & ((j > i - net.window) | (j < net.sinks)))
    start = x.to(torch.bfloat16).double()
    u = torch.nn.functional.layer_norm(start, (net.d,), p["norm_weight"], p["norm_bias"], eps)
    x = x.double()
    for l in range(net.layers):
        qkv = (u @ p[f"{l}.qkv"].T).view(net.tokens, h + 2 * kv, n)
        q, k, v = turned(qkv[:, :h]), turned(qkv[:, h:h + kv]), qkv[:, h + kv:]
        split = lambda a: a.view(net.sequences, net.rows, -1, n).transpose(1, 2)  # noqa: E731
        q, k, v = split(q), split(k).repeat_interleave(h // kv, 1), split(v).repeat_interleave(h // kv, 1)
        o = torch.softmax((q @ k.transpose(-1, -2) / math.sqrt(n)).masked_fill(hidden, -math.inf), -1) @ v
        y = o.transpose(1, 2).reshape(net.tokens, h * n) @ p[f"{l}.out"].T
        x = x + net.alpha * p[f"{l}.a.scale"] * rms(y, p[f"{l}.a.post"])
        u = rms(x, p[f"{l}.a.pre"])
        y = (torch.nn.functional.silu(u @ p[f"{l}.gate"].T) * (u @ p[f"{l}.up"].T)) @ p[f"{l}.down"].T
        x = x + net.alpha * p[f"{l}.b.scale"] * rms(y, p[f"{l}.b.post"])
        u = rms(x, p[f"{l}.b.pre"])
    return u


def test_gradients_of_the_whole_network():
    """Every parameter's gradient against autograd in 64 bits.  On its way a gradient meets at most 20 tensors of each layer that are held in
    bfloat16 (activations, probabilities, gradients), each off by half a step, 2^-8, at most and by 2^-8 / sqrt(3) in the mean square; two layers are 40 of
    them, 2^-8 sqrt(40 / 3) = 0.0143 of a norm when none is amplified; a norm of 4 times that is allowed (products of unit-variance factors
    amplify by up to 2 a layer)."""
    net = _example().Network(layers=2, d=128, f=264, sequences=3, side=9)
    gen = torch.Generator("cuda").manual_seed(3)
    x = torch.empty((net.tokens, net.d), device="cuda").normal_(generator=gen)
    du = torch.empty((net.tokens, net.d), device="cuda").normal_(generator=gen).to(torch.bfloat16)
    out = net.forward(x)
    grads = net.backward(du)
    p = {k: v.double().requires_grad_() for k, v in net.copies.items()}
    want = _definition(net, x, p)
    (want * du.double()).sum().backward()
    bound = 4 * 2.0 ** -8 * math.sqrt(40.0 / 3.0)
    assert ((out.double() - want).norm() / want.norm()).item() <= bound
    for name, g in grads.items():
        ref = p[name].grad
        assert ((g.double() - ref).norm() / ref.norm()).item() <= bound, name


def test_example_runs():
    losses = _example().train(steps=3, workers=2, layers=1, d=64, f=136, sequences=1, side=5)
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses)
