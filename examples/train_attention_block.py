"""A small transformer of windowed attention and gated blocks trained by simulated data-parallel workers.

Every layer projects its normed input, turns queries and keys by their places in a grid (rows and columns), attends within a window and
to a few first tokens, and joins the result to the residual stream with a gate, a scale and the norms on either side; then a gated
feed-forward block, joined in the same way.  A2SGD (Algorithm 1) averages the workers' gradients, AdamW takes the step.  The projections
are plain matrix products.

    python examples/train_attention_block.py [--steps 40] [--workers 2] [--layers 2] [--width 256]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2006_07405_b200 import binding as a2  # noqa: E402

EPS = 1e-5
BF16 = torch.bfloat16


class Network:
    """fp32 weights, their bfloat16 copies, and one worker's activations.  A batch is ``sequences`` grids of ``side`` x ``side`` tokens."""

    def __init__(self, layers, d, f, sequences, side, heads=4, kv_heads=2, head_dim=64, window=40, sinks=3, alpha=0.5, device="cuda", seed=0):
        gen = torch.Generator(device).manual_seed(seed)
        new = lambda *shape, std: torch.empty(shape, device=device).normal_(0.0, std, generator=gen)  # noqa: E731
        ones, zeros = (lambda n: torch.ones(n, device=device)), (lambda n: torch.zeros(n, device=device))
        self.layers, self.d, self.f, self.sequences, self.rows = layers, d, f, sequences, side * side
        self.heads, self.kv_heads, self.head_dim, self.window, self.sinks, self.alpha = heads, kv_heads, head_dim, window, sinks, alpha
        self.tokens = t = sequences * self.rows
        wide = (heads + 2 * kv_heads) * head_dim
        self.params = [("norm_weight", ones(d)), ("norm_bias", zeros(d))]
        for i in range(layers):
            self.params += [(f"{i}.qkv", new(wide, d, std=d ** -0.5)), (f"{i}.out", new(d, heads * head_dim, std=(heads * head_dim) ** -0.5)),
                            (f"{i}.gate", new(f, d, std=d ** -0.5)), (f"{i}.up", new(f, d, std=d ** -0.5)), (f"{i}.down", new(d, f, std=f ** -0.5))]
            for part in ("a", "b"):      # the joins behind the attention and behind the feed-forward block
                self.params += [(f"{i}.{part}.post", 1.0 + new(d, std=0.1)), (f"{i}.{part}.scale", 1.0 + new(1, d, std=0.1)), (f"{i}.{part}.pre", 1.0 + new(d, std=0.1))]
        self.copies = {name: p.to(BF16) for name, p in self.params}
        self.grads = {name: torch.empty_like(c) for name, c in self.copies.items()}
        place = torch.arange(self.rows, device=device, dtype=torch.int32)
        self.positions = torch.stack([place // side, place % side]).repeat(1, sequences).contiguous()
        self.sections = [head_dim // 4, head_dim // 4]
        q = torch.empty((sequences, self.rows, heads, head_dim), dtype=BF16, device=device)
        k = torch.empty((sequences, self.rows, kv_heads, head_dim), dtype=BF16, device=device)
        bytes_ = max(a2.a2sgd_window_attention_workspace(q, k, window, sinks, sequences, backward=True, aligned=True),
                     a2.a2sgd_gated_ffn_workspace(t, d, f, backward=True, aligned=True), a2.a2sgd_residual_norm_workspace(t, d, t),
                     a2.a2sgd_layer_norm_workspace(t, d))
        self.workspace = torch.empty(bytes_, dtype=torch.uint8, device=device)
        self.device = device

    def _new(self, *shape, dtype=BF16):
        return torch.empty(shape, dtype=dtype, device=self.device)

    def _by_sequence(self, x, heads):
        return x.view(self.sequences, self.rows, heads, self.head_dim)

    def _join(self, name):
        c = self.copies
        return dict(kind="rms", post=True, post_weight=c[name + ".post"], gate=c[name + ".scale"], gate_rows=self.tokens, alpha=self.alpha,
                    pre_weight=c[name + ".pre"])

    def _join_forward(self, name, x, y):
        s = {"y": y, "z": self._new(self.tokens, self.d, dtype=torch.float32), "u": self._new(self.tokens, self.d),
             "post": self._new(self.tokens, dtype=torch.float32), "pre": self._new(self.tokens, dtype=torch.float32)}
        a2.a2sgd_residual_norm_forward(x, y, s["z"], s["u"], post_rstd=s["post"], pre_rstd=s["pre"], eps=EPS, **self._join(name))
        return s

    def _join_backward(self, name, s, dz, du):
        dx, dy = self._new(self.tokens, self.d, dtype=torch.float32), self._new(self.tokens, self.d)
        a2.a2sgd_residual_norm_backward(dz, du, s["y"], s["z"], dx, dy, post_rstd=s["post"], pre_rstd=s["pre"], dpost_weight=self.grads[name + ".post"],
                                        dgate=self.grads[name + ".scale"], dpre_weight=self.grads[name + ".pre"], workspace=self.workspace, **self._join(name))
        return dx, dy

    def forward(self, x):
        """x: fp32 [tokens, d]; returns the last normed rows."""
        c, h, kv, n = self.copies, self.heads, self.kv_heads, self.head_dim
        self.saved, self.x0 = [], x
        u, self.mean, self.rstd = self._new(self.tokens, self.d), self._new(self.tokens, dtype=torch.float32), self._new(self.tokens, dtype=torch.float32)
        self.start = x.to(BF16)
        a2.a2sgd_layer_norm_forward(self.start, c["norm_weight"], c["norm_bias"], u, self.mean, self.rstd, EPS)
        for i in range(self.layers):
            s = {"u": u}
            qkv = (u @ c[f"{i}.qkv"].T).view(self.tokens, h + 2 * kv, n)
            s["q"], s["k"], s["v"] = self._new(self.tokens, h, n), self._new(self.tokens, kv, n), qkv[:, h + kv:]
            a2.a2sgd_rotary(qkv[:, :h], qkv[:, h:h + kv], s["q"], s["k"], self.positions, self.sections, ladder_per_axis=True)
            s["o"], s["lse"] = self._new(self.tokens, h, n), self._new(self.sequences, h, self.rows, dtype=torch.float32)
            a2.a2sgd_window_attention_forward(self._by_sequence(s["q"], h), self._by_sequence(s["k"], kv),
                                              s["v"].unflatten(0, (self.sequences, self.rows)), self._by_sequence(s["o"], h), s["lse"],
                                              window=self.window, sinks=self.sinks, workspace=self.workspace)
            s["a"] = self._join_forward(f"{i}.a", x, s["o"].flatten(1) @ c[f"{i}.out"].T)
            y = self._new(self.tokens, self.d)
            s["hidden"], s["gate"], s["up"] = (self._new(self.tokens, self.f) for _ in range(3))
            a2.a2sgd_gated_ffn_forward(s["a"]["u"], c[f"{i}.gate"], c[f"{i}.up"], c[f"{i}.down"], y, s["hidden"], s["gate"], s["up"],
                                       workspace=self.workspace)
            s["b"] = self._join_forward(f"{i}.b", s["a"]["z"], y)
            x, u = s["b"]["z"], s["b"]["u"]
            self.saved.append(s)
        return u

    def backward(self, du):
        """du: bfloat16, the gradient of what ``forward`` returned; returns the parameters' gradients by name, in bfloat16."""
        c, g, h, kv, n = self.copies, self.grads, self.heads, self.kv_heads, self.head_dim
        dz = None
        for i in reversed(range(self.layers)):
            s = self.saved[i]
            dz, dy = self._join_backward(f"{i}.b", s["b"], dz, du)
            du = self._new(self.tokens, self.d)
            a2.a2sgd_gated_ffn_backward(dy, s["a"]["u"], c[f"{i}.gate"], c[f"{i}.up"], c[f"{i}.down"], s["hidden"], s["gate"], s["up"], du,
                                        g[f"{i}.gate"], g[f"{i}.up"], g[f"{i}.down"], workspace=self.workspace)
            dz, dy = self._join_backward(f"{i}.a", s["a"], dz, du)
            g[f"{i}.out"].copy_(dy.T @ s["o"].flatten(1))
            dout = (dy @ c[f"{i}.out"]).view_as(s["o"])
            dqkv = self._new(self.tokens, h + 2 * kv, n)
            dq, dk, dv = dqkv[:, :h], dqkv[:, h:h + kv], dqkv[:, h + kv:]
            grid = lambda t: t.unflatten(0, (self.sequences, self.rows))  # noqa: E731
            a2.a2sgd_window_attention_backward(grid(dout), grid(s["q"]), grid(s["k"]), grid(s["v"]), grid(s["o"]), s["lse"], grid(dq), grid(dk),
                                               grid(dv), window=self.window, sinks=self.sinks, workspace=self.workspace)
            a2.a2sgd_rotary(dq, dk, dq, dk, self.positions, self.sections, ladder_per_axis=True, inverse=True)
            g[f"{i}.qkv"].copy_(dqkv.flatten(1).T @ s["u"])
            du = dqkv.flatten(1) @ c[f"{i}.qkv"]
        a2.a2sgd_layer_norm_backward(du, self.start, c["norm_weight"], self.mean, self.rstd, None, g["norm_weight"], g["norm_bias"], self.workspace)
        return g


def train(steps=40, workers=2, layers=2, d=256, f=512, sequences=2, side=12, lr=1e-3, max_norm=1.0, log=None):
    """Returns the loss before each step (the mean over the workers)."""
    net = Network(layers, d, f, sequences, side)
    params = [p for _, p in net.params]
    like = lambda: [torch.zeros_like(p) for p in params]  # noqa: E731
    # A2SGD over the list of tensors.  Its update w <- w - lr g_hat with w = 0 and lr = -1 leaves the averaged gradient.
    grads, averaged = [like() for _ in range(workers)], like()
    ctx = a2.a2sgd_create(sum(p.numel() for p in params), workers, flags=a2.MODE_ALG1)
    segments = a2.a2sgd_segments_create(ctx, grads, None, averaged)
    n = a2.a2sgd_adamw_state_elements(params)
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    optimiser = a2.a2sgd_adamw_create(params, averaged, m, v, w16=[net.copies[name] for name, _ in net.params])
    norm_and_scale = torch.zeros(2, device="cuda")
    gen = torch.Generator("cuda").manual_seed(1)
    x = [torch.empty((net.tokens, d), device="cuda").normal_(generator=gen) for _ in range(workers)]
    target = [v.roll(1, 0).tanh() for v in x]      # each token's neighbour, which attention has to fetch
    losses = []
    for step in range(1, steps + 1):
        loss = torch.zeros(1, device="cuda")
        for p in range(workers):
            diff = net.forward(x[p]).float() - target[p]
            loss += diff.square().mean() / workers
            g = net.backward((diff * (2.0 / diff.numel())).to(BF16))
            torch._foreach_copy_(grads[p], [g[name] for name, _ in net.params])
        torch._foreach_zero_(averaged)
        a2.a2sgd_step_segments(ctx, segments, lr=-1.0)
        a2.a2sgd_adamw_grad_norm(optimiser, max_norm, norm_and_scale)
        a2.a2sgd_adamw_step(optimiser, lr=lr, step=step, weight_decay=0.01, grad_scale=norm_and_scale[1:])
        losses.append(loss)
        if log and (step % 10 == 0 or step == 1):
            log(f"step {step:4d}  loss {loss.item():.4f}  gradient norm {norm_and_scale[0].item():.4f}")
    losses = torch.cat(losses).tolist()
    for status in (a2.a2sgd_window_attention_status, a2.a2sgd_gated_ffn_status):
        if status() != a2.OK:
            raise a2.A2SGDError(a2.ERR_TIMEOUT, status.__name__)
    optimiser.destroy()
    segments.destroy()
    ctx.destroy()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--workers", type=int, default=2)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--width", type=int, default=256)
    a = ap.parse_args()
    train(a.steps, a.workers, a.layers, a.width, 2 * a.width, log=print)
