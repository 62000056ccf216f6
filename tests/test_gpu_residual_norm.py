"""The residual connection with its gate, scale and norms against its definition in 64 bits, through the binding."""
import math

import pytest
import torch

from paper_2006_07405_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
F32 = 2.0 ** -24
EPS = 1e-5


def rows_of(values, dtype, pad, skew):
    r, c = values.shape
    buf = torch.full((r * (c + pad) + skew,), math.nan, dtype=dtype, device="cuda")
    view = buf.as_strided((r, c), (c + pad, 1), skew)
    view.copy_(values)
    return view


def close(name, got, want, loose):
    """loose: what fp32 arithmetic may be off by before the last rounding."""
    bound = HALF_STEP[got.dtype] * (want.abs() + loose) + loose + TINY[got.dtype]
    over = (got.double() - want).abs() - bound
    assert not torch.isnan(over).any() and over.max().item() <= 0, f"{name}: {over.max().item()} beyond its bound"


class Case:
    def __init__(self, rows, d, kind, post=True, gate_rows=0, dtype="bf16", residual=None, param="f32", pad=0, skew=0, bias=None, weight=True,
                 seed=0, offset=0.0, spread=1.0):
        gen = torch.Generator("cuda").manual_seed(seed)
        normal = lambda *s, std=1.0: torch.empty(s, device="cuda").normal_(0.0, std, generator=gen)  # noqa: E731
        self.kind, self.post, self.gate_rows, self.alpha, self.rows, self.d = kind, post, gate_rows, 0.6, rows, d
        dt, rt, pt = DT[dtype], DT[residual or dtype], DT[param]
        self.dt, self.rt, self.pt = dt, rt, pt
        bias = kind == "layer" if bias is None else bias
        make = lambda v, t: rows_of(v, t, pad, skew)  # noqa: E731
        self.x = make(normal(rows, d) * 2 * spread + offset, rt)
        self.y = make(normal(rows, d) * spread * normal(rows, 1).exp() + normal(1, d) + offset, dt)
        self.dz, self.du = make(normal(rows, d), rt), make(normal(rows, d), dt)
        vector = lambda on, mean: (mean + 0.3 * normal(d)).to(pt) if on else None  # noqa: E731
        self.w1, self.b1 = vector(weight and post, 1.0), vector(bias and post, 0.0)
        self.w2, self.b2 = vector(weight, 1.0), vector(bias, 0.0)
        self.groups = -(-rows // gate_rows) if gate_rows else 0
        self.gate = normal(self.groups, d, std=0.7).to(pt) if gate_rows else None
        new = lambda t: make(torch.full((rows, d), math.nan, device="cuda"), t)  # noqa: E731
        self.z, self.u, self.dx, self.dy = new(rt), new(dt), new(rt), new(dt)
        self.stats = [torch.full((rows,), math.nan, device="cuda") for _ in range(4)]   # post mean, post rstd, pre mean, pre rstd

    def common(self):
        return dict(kind=self.kind, post=self.post, post_weight=self.w1, post_bias=self.b1, gate=self.gate, gate_rows=self.gate_rows,
                    alpha=self.alpha, pre_weight=self.w2, **dict(zip(("post_mean", "post_rstd", "pre_mean", "pre_rstd"), self.stats)))

    def forward(self, z=None, u=None):
        B.a2sgd_residual_norm_forward(self.x, self.y, self.z if z is None else z, self.u if u is None else u, pre_bias=self.b2, eps=EPS,
                                      **self.common())

    def wide(self):
        one = torch.ones(self.d, dtype=torch.float64, device="cuda")
        w = lambda t, other: other if t is None else t.double()  # noqa: E731
        gate = one.expand(self.rows, -1) if self.gate is None else self.gate.double().repeat_interleave(self.gate_rows, 0)[:self.rows]
        return w(self.w1, one), w(self.b1, 0 * one), gate, w(self.w2, one), w(self.b2, 0 * one)

    def norm(self, x, loose):
        """mean, rstd, normalised rows, and the bounds of the three: fp32 sums of d terms in runs and trees (at most 40 roundings deep),
        the division, root and reciprocal; loose is what x itself may be off by."""
        mean = x.mean(1, keepdim=True) if self.kind == "layer" else torch.zeros((self.rows, 1), dtype=torch.float64, device="cuda")
        c = x - mean
        var = c.square().mean(1, keepdim=True) + EPS
        rstd = var.rsqrt()
        m_off = 40 * F32 * x.abs().mean(1, keepdim=True) + loose.mean(1, keepdim=True) if self.kind == "layer" else 0 * mean
        c_off = loose + m_off + 2 * F32 * x.abs()
        r_off = rstd * (40 * F32 + (c.abs() * c_off).mean(1, keepdim=True) / var + (c_off.square()).mean(1, keepdim=True) / var)
        hat = c * rstd
        return mean, rstd, hat, m_off, r_off, c_off * rstd + c.abs() * r_off + 3 * F32 * hat.abs()

    def check_forward(self):
        w1, b1, gate, w2, b2 = self.wide()
        y, x = self.y.double(), self.x.double()
        zero = torch.zeros_like(y)
        n, n_off = y, zero
        if self.post:
            mean, rstd, hat, m_off, r_off, h_off = self.norm(y, zero)
            close("post rstd", self.stats[1], rstd[:, 0], r_off[:, 0])
            if self.kind == "layer":
                close("post mean", self.stats[0], mean[:, 0], m_off[:, 0])
            n, n_off = hat * w1 + b1, h_off * w1.abs() + 4 * F32 * ((hat * w1).abs() + b1.abs())
        z = x + self.alpha * gate * n
        z_off = self.alpha * gate.abs() * (n_off + 4 * F32 * n.abs()) + 2 * F32 * (x.abs() + z.abs())
        close("z", self.z, z, z_off)
        mean, rstd, hat, m_off, r_off, h_off = self.norm(z, z_off)
        close("pre rstd", self.stats[3], rstd[:, 0], r_off[:, 0])
        if self.kind == "layer":
            close("pre mean", self.stats[2], mean[:, 0], m_off[:, 0])
        close("u", self.u, hat * w2 + b2, h_off * w2.abs() + 4 * F32 * ((hat * w2).abs() + b2.abs()))

    def backward(self, dz=True, dx=None, dy=None, sums=True):
        pt = self.pt
        new = lambda n: torch.full((n,), math.nan, dtype=pt, device="cuda")  # noqa: E731
        self.sums = {"dpre_weight": new(self.d), "dpre_bias": new(self.d)}
        if self.post:
            self.sums.update(dpost_weight=new(self.d), dpost_bias=new(self.d))
        if self.gate is not None:
            self.sums["dgate"] = new(self.groups * self.d).view(self.groups, self.d)
        n = B.a2sgd_residual_norm_workspace(self.rows, self.d, self.gate_rows)
        work = torch.full((n + 256,), 0xAB, dtype=torch.uint8, device="cuda")
        B.a2sgd_residual_norm_backward(self.dz if dz else None, self.du, self.y, self.z, self.dx if dx is None else dx,
                                       self.dy if dy is None else dy, workspace=work[:n], **self.common(), **(self.sums if sums else {}))
        torch.cuda.synchronize()
        assert (work[n:] == 0xAB).all()

    def check_backward(self, dz=True):
        w1, b1, gate, w2, _ = self.wide()
        layer, d = self.kind == "layer", self.d
        mean1, rstd1, mean2, rstd2 = (s.double()[:, None] for s in self.stats)
        if not layer:
            mean1, mean2 = torch.zeros_like(rstd2), torch.zeros_like(rstd2)

        def back(g, g_off, a, mean, rstd):
            hat = (a - mean) * rstd
            h_off = 3 * F32 * rstd * (a.abs() + mean.abs())
            s0, s1 = g.mean(1, keepdim=True), (g * hat).mean(1, keepdim=True)
            s0_off = 40 * F32 * g.abs().mean(1, keepdim=True) + g_off.mean(1, keepdim=True)
            s1_off = 40 * F32 * (g * hat).abs().mean(1, keepdim=True) + (g_off * hat.abs() + g.abs() * h_off).mean(1, keepdim=True)
            if not layer:
                s0, s0_off = 0 * s0, 0 * s0_off
            off = rstd * (g_off + s0_off + hat.abs() * s1_off + s1.abs() * h_off + 5 * F32 * (g.abs() + s0.abs() + (hat * s1).abs()))
            return hat, h_off, (g - s0 - hat * s1) * rstd, off

        du, y, z = self.du.double(), self.y.double(), self.z.double()
        hat2, h2_off, t, t_off = back(du * w2, 2 * F32 * (du * w2).abs(), z, mean2, rstd2)
        if dz:
            t = t + self.dz.double()
            t_off = t_off + 2 * F32 * t.abs()
        close("dx", self.dx, t, t_off)
        # sums over the rows: in runs of a CTA, the gates', and eight strips
        deep = (self.rows / 100 + 60) * F32
        total = lambda v, off: (v.sum(0), off.sum(0) + deep * v.abs().sum(0))  # noqa: E731
        close("dpre_weight", self.sums["dpre_weight"], *total(du * hat2, du.abs() * h2_off))
        close("dpre_bias", self.sums["dpre_bias"], *total(du, 0 * du))
        dn = self.alpha * gate * t
        dn_off = self.alpha * gate.abs() * (t_off + 3 * F32 * t.abs())
        n, n_off = y, 0 * y
        if self.post:
            hat1, h1_off, dy, dy_off = back(dn * w1, dn_off * w1.abs() + 2 * F32 * (dn * w1).abs(), y, mean1, rstd1)
            close("dpost_weight", self.sums["dpost_weight"], *total(dn * hat1, dn_off * hat1.abs() + dn.abs() * h1_off))
            close("dpost_bias", self.sums["dpost_bias"], *total(dn, dn_off))
            n, n_off = hat1 * w1 + b1, h1_off * w1.abs() + 3 * F32 * ((hat1 * w1).abs() + b1.abs())
        else:
            dy, dy_off = dn, dn_off
        close("dy", self.dy, dy, dy_off)
        if self.gate is not None:
            each, off = self.alpha * t * n, self.alpha * (t_off * n.abs() + t.abs() * (n_off + 4 * F32 * (n.abs() + b1.abs())))
            for g in range(self.groups):
                cut = slice(g * self.gate_rows, (g + 1) * self.gate_rows)
                value, loose = total(each[cut], off[cut])
                close(f"dgate {g}", self.sums["dgate"][g], value, loose + deep * ((t * self.alpha * (n - b1)).abs() + (t * self.alpha * b1).abs())[cut].sum(0))


def both(**kw):
    c = Case(**kw)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()
    return c


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dtype, residual, param", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("bf16", "f32", "f32"), ("f16", "f16", "f32"), ("f16", "f32", "f16")])
@pytest.mark.parametrize("rows, d", [(1, 8), (5, 1600), (300, 264), (40, 33)])
def test_types(kind, dtype, residual, param, rows, d):
    both(rows=rows, d=d, kind=kind, dtype=dtype, residual=residual, param=param, gate_rows=max(1, rows // 3))


@pytest.mark.parametrize("d", [1, 2, 7, 31, 32, 255, 256, 257, 1001, 2048, 2056, 4096, 4104, 5000, 5001, 8192])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_widths(kind, d):
    both(rows=9, d=d, kind=kind, gate_rows=4, residual="f32")


@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("gate_rows", [0, 1, 2, 7, 100, 1000, 5000])
def test_gates(post, gate_rows):
    both(rows=1000, d=96, kind="layer", post=post, gate_rows=gate_rows)


@pytest.mark.parametrize("rows", [1, 2, 147, 149, 3000, 20011])
def test_rows(rows):
    both(rows=rows, d=40, kind="rms", gate_rows=max(1, rows // 5), residual="f32")


@pytest.mark.parametrize("pad, skew", [(0, 1), (3, 0), (8, 8), (5, 2)])
def test_strides_and_addresses(pad, skew):
    both(rows=30, d=128, kind="layer", gate_rows=11, pad=pad, skew=skew)
    both(rows=30, d=128, kind="rms", gate_rows=11, pad=pad, skew=skew, residual="f32")


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_without_parameters(kind):
    both(rows=30, d=64, kind=kind, weight=False, bias=False)
    both(rows=30, d=64, kind=kind, weight=True, bias=kind == "rms")
    both(rows=30, d=64, kind=kind, weight=False, bias=True, post=False)


def test_rows_far_from_zero():
    """A mean of 1000 deviations: squares about anything else would lose the variance."""
    both(rows=20, d=1600, kind="layer", dtype="f32", offset=1000.0)


def test_constant_rows():
    c = Case(rows=4, d=64, kind="layer", dtype="f32")
    c.y.fill_(3.0)
    c.x.fill_(-2.0)
    c.b1.fill_(0.5)
    c.forward()
    c.check_forward()


def test_in_place_and_left_out():
    c = both(rows=50, d=200, kind="layer", gate_rows=20)
    z, u = c.z.clone(), c.u.clone()
    x, y = c.x.clone(), c.y.clone()
    c.forward(z=c.x, u=c.y)
    assert torch.equal(c.x, z) and torch.equal(c.y, u)
    c.x.copy_(x)
    c.y.copy_(y)
    dx, dy, sums, dz, du = c.dx.clone(), c.dy.clone(), c.sums, c.dz.clone(), c.du.clone()
    c.backward(dx=c.dz, dy=c.du)
    assert torch.equal(c.dz, dx) and torch.equal(c.du, dy) and all(torch.equal(sums[k], c.sums[k]) for k in sums)
    c.dz.copy_(dz)
    c.du.copy_(du)
    c.backward(dz=False)
    c.check_backward(dz=False)
    # without the sums, and each sum by itself
    c.backward(sums=False)
    assert torch.isnan(c.sums["dpre_weight"]).all()
    work = torch.empty(B.a2sgd_residual_norm_workspace(50, 200, 20), dtype=torch.uint8, device="cuda")
    for name in sums:
        one = torch.full_like(sums[name], math.nan)
        B.a2sgd_residual_norm_backward(dz, du, c.y, c.z, None, None, workspace=work, **c.common(), **{name: one})
        assert torch.equal(one, sums[name])


def test_gradients_by_differences():
    c = Case(rows=12, d=48, kind="layer", gate_rows=5, dtype="f32")
    c.forward()
    c.backward()
    gen = torch.Generator("cuda").manual_seed(7)
    layer = lambda v: (v - v.mean(1, keepdim=True)) * (v.var(1, correction=0, keepdim=True) + EPS).rsqrt()  # noqa: E731

    def loss(x, y, w1, b1, gate, w2, b2):
        z = x + c.alpha * gate.repeat_interleave(5, 0)[:12] * (layer(y) * w1 + b1)
        return ((layer(z) * w2 + b2) * c.du.double()).sum().item() + (z * c.dz.double()).sum().item()

    at = [t.double() for t in (c.x, c.y, c.w1, c.b1, c.gate, c.w2, c.b2)]
    grads = (c.dx, c.dy, c.sums["dpost_weight"], c.sums["dpost_bias"], c.sums["dgate"], c.sums["dpre_weight"], c.sums["dpre_bias"])
    for i, g in enumerate(grads):
        step = torch.empty(at[i].shape, dtype=torch.float64, device="cuda").normal_(generator=gen)
        plus, minus = list(at), list(at)
        plus[i], minus[i] = at[i] + 1e-5 * step, at[i] - 1e-5 * step
        want = (loss(*plus) - loss(*minus)) / 2e-5
        # fp32 arithmetic: 200 half steps of every term; the difference itself: its third derivative's 1e-10
        slack = 200 * F32 * (g.double() * step).abs().sum().item() + 1e-6 * (1 + abs(want))
        assert abs((g.double() * step).sum().item() - want) <= slack, i


def test_twice_the_same_bits_and_captured():
    c = both(rows=700, d=1600, kind="rms", gate_rows=128, residual="f32")
    first = [t.clone() for t in (c.z, c.u, c.dx, c.dy, *c.sums.values())]
    work = torch.empty(B.a2sgd_residual_norm_workspace(700, 1600, 128), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward()
        B.a2sgd_residual_norm_backward(c.dz, c.du, c.y, c.z, c.dx, c.dy, workspace=work, **c.common(), **c.sums)
    for t in (c.z, c.u, c.dx, c.dy, *c.sums.values()):
        t.fill_(math.nan)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, (c.z, c.u, c.dx, c.dy, *c.sums.values())))


def test_no_rows():
    c = Case(rows=0, d=64, kind="layer")
    c.forward()
    c.backward()
    assert not any(t.any() for t in c.sums.values())


def test_refusals():
    c = Case(rows=6, d=64, kind="layer", gate_rows=3)
    base = dict(c.common(), x=c.x, y=c.y, z=c.z, u=c.u)
    go = lambda **kw: B.a2sgd_residual_norm_forward(**{**base, **kw})  # noqa: E731
    go()
    for bad in (dict(kind="group"), dict(gate_rows=0), dict(gate=c.gate[:1]), dict(post_weight=c.w1.half()), dict(z=c.z[:3]), dict(y=c.y[0]),
                dict(u=c.u.float()), dict(pre_mean=torch.empty(5, device="cuda")), dict(x=c.x.double(), z=c.z.double()), dict(x=c.x.cpu())):
        with pytest.raises(ValueError):
            go(**bad)
    for bad in (dict(eps=-1.0), dict(eps=math.nan), dict(alpha=math.inf), dict(x=c.x.half(), z=c.z.half())):
        with pytest.raises(B.A2SGDError) as e:
            go(**bad)
        assert e.value.status == B.ERR_ARG
    wide = torch.zeros((1, 8200), device="cuda")
    with pytest.raises(B.A2SGDError) as e:
        B.a2sgd_residual_norm_forward(wide, wide, torch.empty_like(wide), torch.empty_like(wide))
    assert e.value.status == B.ERR_TOO_LARGE
    back = dict(c.common(), dz=c.dz, du=c.du, y=c.y, z=c.z, dx=c.dx, dy=c.dy)
    for bad in (dict(pre_rstd=None), dict(pre_mean=None), dict(post_rstd=None), dict(post_mean=None), dict(dpre_weight=torch.empty(64, device="cuda")),
                dict(post=False, dpost_weight=torch.empty(64, device="cuda"), workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(B.A2SGDError) as e:
            B.a2sgd_residual_norm_backward(**{**back, **bad})
        assert e.value.status == B.ERR_ARG
