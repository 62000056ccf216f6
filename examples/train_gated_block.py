"""A small residual network of gated blocks trained by simulated data-parallel workers, all of it on the library's kernels.

Every worker runs ``x <- x + ffn(layer_norm(x))`` over its share of a batch and back; A2SGD (Algorithm 1) turns the
workers' gradients into one averaged gradient for each tensor; its global norm is clipped and AdamW takes the step, in fp32
or with 8-bit states, and writes the bfloat16 weights that the next forward pass reads.

    python examples/train_gated_block.py [--steps 60] [--state-bits 8] [--workers 4] [--layers 2] [--width 256]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2006_07405_b200 import binding as a2  # noqa: E402

EPS = 1e-5
NAMES = ("norm_weight", "norm_bias", "w_gate", "w_up", "w_down")


class Network:
    """fp32 weights, their bfloat16 copies, and the activations of one worker's pass."""

    def __init__(self, layers, d, f, tokens, device="cuda", seed=0):
        gen = torch.Generator(device).manual_seed(seed)
        new = lambda *shape, std: torch.empty(shape, device=device).normal_(0.0, std, generator=gen)  # noqa: E731
        self.layers, self.d, self.f, self.tokens = layers, d, f, tokens
        self.params = []
        for _ in range(layers):
            self.params += [torch.ones(d, device=device), torch.zeros(d, device=device), new(f, d, std=d ** -0.5),
                            new(f, d, std=d ** -0.5), new(d, f, std=f ** -0.5)]
        self.copies = [p.to(torch.bfloat16) for p in self.params]
        rows = lambda c: torch.empty((tokens, c), dtype=torch.bfloat16, device=device)  # noqa: E731
        stat = lambda: torch.empty(tokens, device=device)  # noqa: E731
        self.saved = [{"x": None, "normed": rows(d), "mean": stat(), "rstd": stat(), "hidden": rows(f), "gate": rows(f),
                       "up": rows(f)} for _ in range(layers)]
        self.grads16 = [torch.empty_like(c) for c in self.copies]
        bytes_ = max(a2.a2sgd_gated_ffn_workspace(tokens, d, f, backward=True, aligned=True),
                     a2.a2sgd_layer_norm_workspace(tokens, d))
        self.workspace = torch.empty(bytes_, dtype=torch.uint8, device=device)

    def _layer(self, i):
        return dict(zip(NAMES, self.copies[5 * i:5 * i + 5]))

    def forward(self, x):
        for i, s in enumerate(self.saved):
            p, s["x"], y = self._layer(i), x, torch.empty_like(x)
            a2.a2sgd_layer_norm_forward(x, p["norm_weight"], p["norm_bias"], s["normed"], s["mean"], s["rstd"], EPS)
            a2.a2sgd_gated_ffn_forward(s["normed"], p["w_gate"], p["w_up"], p["w_down"], y, s["hidden"], s["gate"], s["up"],
                                       workspace=self.workspace)
            x = x + y
        return x

    def backward(self, dout):
        """The gradients of the last forward pass, in bfloat16, one for each parameter."""
        for i in reversed(range(self.layers)):
            s, p = self.saved[i], self._layer(i)
            dnorm_w, dnorm_b, dw_gate, dw_up, dw_down = self.grads16[5 * i:5 * i + 5]
            dnormed, dx = torch.empty_like(dout), torch.empty_like(dout)
            a2.a2sgd_gated_ffn_backward(dout, s["normed"], p["w_gate"], p["w_up"], p["w_down"], s["hidden"], s["gate"],
                                        s["up"], dnormed, dw_gate, dw_up, dw_down, workspace=self.workspace)
            a2.a2sgd_layer_norm_backward(dnormed, s["x"], p["norm_weight"], s["mean"], s["rstd"], dx, dnorm_w, dnorm_b,
                                         self.workspace)
            dout = dout + dx
        return self.grads16


def train(steps=60, workers=4, layers=2, d=256, f=512, tokens=256, state_bits=32, lr=3e-3, max_norm=1.0, log=None):
    """Returns the loss before each step (the mean over the workers)."""
    net = Network(layers, d, f, tokens)
    params, count = net.params, sum(p.numel() for p in net.params)
    like = lambda: [torch.zeros_like(p) for p in params]  # noqa: E731

    # A2SGD over the list of tensors.  Its update w <- w - lr g_hat with w = 0 and lr = -1 leaves the averaged gradient.
    grads, averaged = [like() for _ in range(workers)], like()
    ctx = a2.a2sgd_create(count, workers, flags=a2.MODE_ALG1)
    segments = a2.a2sgd_segments_create(ctx, grads, None, averaged)

    n = a2.a2sgd_adamw_state_elements(params)
    zeros = lambda k, dtype=torch.float32: torch.zeros(k, dtype=dtype, device="cuda")  # noqa: E731
    if state_bits == 8:
        state = (zeros(n, torch.int8), zeros(n, torch.uint8), zeros(n // a2.ADAMW_BLOCK), zeros(n // a2.ADAMW_BLOCK))
    else:
        state = (zeros(n), zeros(n), None, None)
    optimiser = a2.a2sgd_adamw_create(params, averaged, *state, w16=net.copies)
    norm_and_scale = zeros(2)

    # a fixed batch for each worker, and the map to learn
    gen = torch.Generator("cuda").manual_seed(1)
    x = [torch.empty((tokens, d), device="cuda").normal_(generator=gen).to(torch.bfloat16) for _ in range(workers)]
    turn = torch.empty((d, d), device="cuda").normal_(0.0, d ** -0.5, generator=gen)
    target = [(v.float() @ turn).tanh() for v in x]

    losses = []
    for step in range(1, steps + 1):
        loss = zeros(1)
        for p in range(workers):
            diff = net.forward(x[p]).float() - target[p]
            loss += diff.square().mean() / workers
            torch._foreach_copy_(grads[p], net.backward((diff * (2.0 / diff.numel())).to(torch.bfloat16)))
        torch._foreach_zero_(averaged)
        a2.a2sgd_step_segments(ctx, segments, lr=-1.0)
        a2.a2sgd_adamw_grad_norm(optimiser, max_norm, norm_and_scale)
        a2.a2sgd_adamw_step(optimiser, lr=lr, step=step, weight_decay=0.01, grad_scale=norm_and_scale[1:])
        losses.append(loss)
        if log and (step % 10 == 0 or step == 1):
            log(f"step {step:4d}  loss {loss.item():.4f}  gradient norm {norm_and_scale[0].item():.4f}")
    losses = torch.cat(losses).tolist()
    if a2.a2sgd_gated_ffn_status() != a2.OK:
        raise a2.A2SGDError(a2.ERR_TIMEOUT, "a2sgd_gated_ffn")
    optimiser.destroy()
    segments.destroy()
    ctx.destroy()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=32)
    a = ap.parse_args()
    train(a.steps, a.workers, a.layers, a.width, 2 * a.width, state_bits=a.state_bits, log=print)
