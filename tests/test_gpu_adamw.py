"""AdamW over a list of tensors (32- and 8-bit states) and the gradients' norm, through the binding.

References: the formulas in 64 bits, and for the 8-bit codes the same sequence of single-precision
operations in numpy, which fixes them to the bit.

Tolerances.  One fp32 rounding is u = 2^-24 of its result.  m and v are two products (v three) and a sum: at
most 3 u (4 u) of the terms' absolute sum; the coefficients add one u each, so 5 u and 6 u.  w: the decay
product and the final difference 3 u |w|; the update m / (sqrt(v) root + eps) * rate carries the relative errors
of m (bounded by the above), sqrt(v), the sum, the quotient, the product and the coefficients: 16 u of the largest
possible update, (|b1 m| + |(1 - b1) g|) in place of |m|."""
import math

import numpy as np
import pytest
import torch

from paper_2006_07405_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)
F32 = np.float32


def _starts(numel):
    at, out = 0, []
    for n in numel:
        out.append(at)
        at += -(-n // 256) * 256
    return out, at


class Problem:
    """Tensors cut out of wider buffers, so that writes outside of them show."""

    def __init__(self, numel, gtype=torch.float32, skew=0, bits=32, copy=None, seed=0, gscale=1e-2):
        gen = torch.Generator("cuda").manual_seed(seed)
        rnd = lambda n, s: torch.empty(n, device="cuda").normal_(0, s, generator=gen)  # noqa: E731
        self.numel = numel
        gap = 64
        total = sum(-(-n // 64) * 64 + gap for n in numel) + gap
        self.wbuf = torch.full((total,), 7.0, device="cuda")
        self.gbuf = torch.full((total,), 5.0, device="cuda").to(gtype)
        self.cbuf = torch.full((total,), 3.0, device="cuda").to(copy) if copy else None
        self.w, self.g, self.c, self.inside = [], [], [], torch.zeros(total, dtype=torch.bool, device="cuda")
        at = gap // 2 * 2
        for n in numel:
            lo = at + skew
            self.wbuf[lo:lo + n] = rnd(n, 0.5)
            self.gbuf[lo:lo + n] = (rnd(n, gscale)).to(gtype)
            self.w.append(self.wbuf[lo:lo + n])
            self.g.append(self.gbuf[lo:lo + n])
            if copy:
                self.c.append(self.cbuf[lo:lo + n])
            self.inside[lo:lo + n] = True
            at += -(-n // 64) * 64 + gap
        self.starts, self.n = _starts(numel)
        live = torch.zeros(self.n, device="cuda")
        for s, n in zip(self.starts, numel):
            live[s:s + n] = 1
        m, r = rnd(self.n, gscale).mul_(live), rnd(self.n, 0.3).exp_().mul_(gscale).mul_(live)
        self.ms = self.vs = None
        if bits == 32:
            self.m, self.v = m, r * r
        else:
            self.ms = m.view(-1, 256).abs().amax(1)
            self.vs = r.view(-1, 256).amax(1)
            self.m = ((m.view(-1, 256).abs() / self.ms[:, None].clamp_min(1e-30)).sqrt() * 127).round().mul(
                m.view(-1, 256).sign()).to(torch.int8).view(-1)
            self.v = ((r.view(-1, 256) / self.vs[:, None].clamp_min(1e-30)).sqrt() * 255).round().clamp_min(2).to(torch.uint8).view(-1)
        self.plan = B.a2sgd_adamw_create(self.w, self.g, self.m, self.v, self.ms, self.vs, self.c if copy else None)

    def flat(self, parts):
        """Tensors in the state's layout, zero between them, fp64 numpy."""
        out = np.zeros(self.n)
        for s, t in zip(self.starts, parts):
            out[s:s + t.numel()] = t.double().cpu().numpy()
        return out


def _formula(w, g, m, v, step, lr, beta1, beta2, eps, weight_decay):
    m2, v2 = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    denom = np.sqrt(v2) / math.sqrt(1 - beta2 ** step) + eps
    rate = lr / (1 - beta1 ** step)
    w2 = w * (1 - lr * weight_decay) - rate * m2 / denom
    tol_m = 5 * U * (beta1 * np.abs(m) + (1 - beta1) * np.abs(g)) + 1e-44
    tol_v = 6 * U * v2 + 1e-44
    tol_w = 3 * U * np.abs(w) + 16 * U * rate * (beta1 * np.abs(m) + (1 - beta1) * np.abs(g)) / denom + 1e-44
    return (w2, tol_w), (m2, tol_m), (v2, tol_v)


LISTS = [[1], [255], [256], [257], [2048], [2049], [5, 1, 256, 3000, 8, 70001], [1 << 18]]


@pytest.mark.parametrize("numel", LISTS, ids=lambda x: "x".join(map(str, x)))
@pytest.mark.parametrize("gtype,skew,copy", [(torch.float32, 0, None), (torch.float32, 1, torch.bfloat16),
                                             (torch.bfloat16, 0, torch.bfloat16), (torch.float16, 3, torch.float16),
                                             (torch.bfloat16, 4, None)])
def test_step_with_32_bit_states(numel, gtype, skew, copy):
    p = Problem(numel, gtype, skew, 32, copy)
    scale = torch.tensor([0.5], device="cuda")
    for step in (1, 2, 1000):
        w, g, m, v = p.flat(p.w), p.flat(p.g) * 0.5, p.m.double().cpu().numpy(), p.v.double().cpu().numpy()
        B.a2sgd_adamw_step(p.plan, step=step, grad_scale=scale, **HYPER)
        for (ref, tol), got in zip(_formula(w, g, m, v, step, **HYPER), (p.flat(p.w), p.m.double().cpu().numpy(), p.v.double().cpu().numpy())):
            assert np.all(np.abs(got - ref) <= tol)
        if copy:
            for a, b in zip(p.c, p.w):
                assert torch.equal(a, b.to(copy))
    assert torch.all(p.wbuf[~p.inside] == 7.0) and torch.all(p.gbuf[~p.inside] == 5.0)
    if copy:
        assert torch.all(p.cbuf[~p.inside] == 3.0)


def _hash(places, step):
    with np.errstate(over="ignore"):
        h = places.astype(np.uint32) * np.uint32(0x9E3779B1) + np.uint32((step * 0x85A308D3 + 0x243F6A89) & 0xFFFFFFFF)
        h ^= h >> np.uint32(16)
        h *= np.uint32(0x7FEB3525)
        h ^= h >> np.uint32(15)
        h *= np.uint32(0x94D049BB)
        h ^= h >> np.uint32(16)
    return (h >> np.uint32(20)).astype(F32), ((h >> np.uint32(8)) & np.uint32(0xFFF)).astype(F32)


def _codes(x, top, u):
    scale = x.max(axis=1, keepdims=True)
    scale = np.where(scale < F32(2.0 ** -100), F32(0), scale)
    with np.errstate(divide="ignore"):
        gain = np.where(scale > 0, (F32(1) / scale) * F32(top * top), F32(0)).astype(F32)
    s = x * gain
    q = np.floor(np.sqrt(s))
    q = q + (s - q * q > u.reshape(x.shape) * F32(1 / 4096) * (F32(2) * q + F32(1))).astype(F32)
    return np.minimum(q, F32(top)), scale


def _step8(w, g, mq, vq, ms, vs, step, lr, beta1, beta2, eps, weight_decay):
    """The header's sequence of single-precision operations."""
    q, a, b = mq.astype(F32).reshape(-1, 256), ms.reshape(-1, 1), vs.reshape(-1, 1)
    m = (q * np.abs(q)) * (a * F32(1 / 16129))
    q = vq.astype(F32).reshape(-1, 256)
    r = (q * q) * (b * F32(1 / 65025))
    v = r * r
    g, w = g.reshape(-1, 256), w.reshape(-1, 256)
    m = m * F32(beta1) + g * F32(1 - beta1)
    v = v * F32(beta2) + (g * g) * F32(1 - beta2)
    r = np.sqrt(v)
    d = r * F32(1 / math.sqrt(1 - beta2 ** step)) + F32(eps)
    w = w * F32(1 - lr * weight_decay) - (m / d) * F32(lr / (1 - beta1 ** step))
    um, ur = _hash(np.arange(m.size, dtype=np.uint64), step)
    qm, ms = _codes(np.abs(m), 127, um)
    qr, vs = _codes(r, 255, ur)
    return w.reshape(-1), np.where(m < 0, -qm, qm).reshape(-1), np.maximum(qr, F32(2)).reshape(-1), ms.reshape(-1), vs.reshape(-1)


@pytest.mark.parametrize("numel", LISTS, ids=lambda x: "x".join(map(str, x)))
@pytest.mark.parametrize("gtype,skew,copy", [(torch.float32, 0, None), (torch.bfloat16, 0, torch.bfloat16),
                                             (torch.float16, 1, None), (torch.float32, 2, torch.float16)])
def test_step_with_8_bit_states_is_defined_to_the_bit(numel, gtype, skew, copy):
    p = Problem(numel, gtype, skew, 8, copy)
    for step in (1, 2, 77):
        w, g = p.flat(p.w).astype(F32), p.flat(p.g).astype(F32)
        state = [t.cpu().numpy() for t in (p.m, p.v, p.ms, p.vs)]
        B.a2sgd_adamw_step(p.plan, step=step, **HYPER)
        ref = _step8(w, g, *state, step, **HYPER)
        live = p.flat([torch.ones(n) for n in numel]) > 0
        assert np.array_equal(p.flat(p.w).astype(F32)[live], ref[0][live])
        for got, want in zip((p.m, p.v, p.ms, p.vs), ref[1:]):
            assert np.array_equal(got.cpu().numpy().astype(F32), want)
        if copy:
            for a, b in zip(p.c, p.w):
                assert torch.equal(a, b.to(copy))
    assert torch.all(p.wbuf[~p.inside] == 7.0)


def test_8_bit_states_stay_within_a_code_of_the_formula():
    """64-bit formula from the values that the codes stand for: w to rounding, m and sqrt(v) within one code.
    The codes are squares, so the one next to q is (2 q + 1) / top^2 of the scale away, and at least one."""
    p = Problem([70_001], seed=3, bits=8)
    m, v = torch.empty(p.n, device="cuda"), torch.empty(p.n, device="cuda")
    B.a2sgd_adamw_read_state(p.plan, m, v)
    old = [t.double().cpu().numpy() for t in (m, v)]
    w, g = p.flat(p.w), p.flat(p.g)
    B.a2sgd_adamw_step(p.plan, step=5, **HYPER)
    (w2, tol_w), (m2, _), (v2, _) = _formula(w, g, *old, 5, **HYPER)
    assert np.all(np.abs(p.flat(p.w) - w2) <= tol_w)
    B.a2sgd_adamw_read_state(p.plan, m, v)
    ms, vs = (np.repeat(t.double().cpu().numpy(), 256) for t in (p.ms, p.vs))
    for got, ref, scale, top, low in ((m.double().cpu().numpy(), m2, ms, 127, 0), (v.double().sqrt().cpu().numpy(), np.sqrt(v2), vs, 255, 4)):
        q = np.sqrt(np.abs(ref) / scale) * top
        assert np.all(np.abs(got - ref) <= np.maximum(2 * q + 1, low) / top ** 2 * scale * (1 + 1e-5))


def test_8_bit_second_moment_decays_when_gradients_fall_silent():
    """With no gradient v falls by beta2 a step, 0.05 % of sqrt(v), a fraction of a code; the dither makes the mean of
    many elements follow.  200 steps: 0.9048 for sqrt(v).  A step moves the code of an element (q near 200) by about
    p = 0.05 of one, variance p (1 - p) codes^2, so after 200 steps the deviation is under sqrt(200 * 0.05) = 3.2 of
    200 codes, 3.2 % of sqrt(v), and over 65536 elements of 1e-4; the block's scale, its largest value, drifts upwards
    against the others by about three deviations, but the values do not depend on it.  Allowed: 0.01."""
    n = 65536
    p = Problem([n], bits=8)
    p.g[0].zero_()
    m0, v0 = torch.zeros(n, device="cuda"), torch.empty(n, device="cuda").uniform_(0.5, 1.0)
    B.a2sgd_adamw_write_state(p.plan, m0, v0)
    B.a2sgd_adamw_read_state(p.plan, m0, v0)
    before = v0.double().sqrt().mean().item()
    for step in range(1, 201):
        B.a2sgd_adamw_step(p.plan, step=step, **HYPER)
    B.a2sgd_adamw_read_state(p.plan, m0, v0)
    assert abs(v0.double().sqrt().mean().item() / before - 0.999 ** 100) < 0.01
    assert torch.all(m0 == 0)


def test_state_export_and_import():
    """Import rounds to the nearer square: within half the distance to the next code."""
    p = Problem([1000, 33], bits=8, seed=9)
    gen = torch.Generator("cuda").manual_seed(1)
    m = torch.empty(p.n, device="cuda").normal_(0, 1e-3, generator=gen)
    r = torch.empty(p.n, device="cuda").normal_(0, 0.5, generator=gen).exp_()
    B.a2sgd_adamw_write_state(p.plan, m, r * r)
    m2, v2 = torch.empty_like(m), torch.empty_like(m)
    B.a2sgd_adamw_read_state(p.plan, m2, v2)
    for got, ref, top, low in ((m2, m, 127, 0), (v2.sqrt(), r, 255, 4)):
        got, ref = got.double().view(-1, 256), ref.double().view(-1, 256)
        scale = ref.abs().amax(1, keepdim=True)
        q = (ref.abs() / scale).sqrt() * top
        assert torch.all((got - ref).abs() <= ((q + 0.5).clamp_min(low) + 1e-3) / top ** 2 * scale)
    # 32-bit plans copy
    p = Problem([1000, 33], bits=32, seed=9)
    B.a2sgd_adamw_write_state(p.plan, m, v2)
    assert torch.equal(p.m, m) and torch.equal(p.v, v2)
    B.a2sgd_adamw_read_state(p.plan, m2, None)
    assert torch.equal(m2, m)


@pytest.mark.parametrize("bits", [32, 8])
def test_zero_and_tiny_blocks(bits):
    """Gradients of zero leave zero states and only decay w; a block below 2^-100 is held as zeros in 8 bits."""
    p = Problem([512, 256], bits=bits)
    for t in (p.m, p.v, p.ms, p.vs):
        if t is not None:
            t.zero_()
    p.g[0].zero_()
    p.g[1].fill_(1e-32)
    w = [t.clone() for t in p.w]
    B.a2sgd_adamw_step(p.plan, step=1, **HYPER)
    assert torch.equal(p.w[0], w[0] * F32(1 - HYPER["lr"] * HYPER["weight_decay"]))
    m, v = torch.empty(p.n, device="cuda"), torch.empty(p.n, device="cuda")
    B.a2sgd_adamw_read_state(p.plan, m, v)
    assert torch.all(m[:512] == 0) and torch.all(v[:512] == 0)
    assert torch.all(torch.isfinite(m)) and torch.all(torch.isfinite(v)) and torch.all(torch.isfinite(p.w[1]))
    if bits == 8:
        assert torch.all(m == 0) and torch.all(v == 0)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_gradient_that_is_not_finite(bits, bad):
    """It shows in its own element (32 bits) or block (8 bits) and nowhere else."""
    p, q = Problem([1000, 300], bits=bits, seed=4), Problem([1000, 300], bits=bits, seed=4)
    p.g[0][300] = bad
    for x in (p, q):
        B.a2sgd_adamw_step(x.plan, step=1, **HYPER)
    assert not torch.isfinite(p.w[0][300])
    keep = torch.ones(1000, dtype=torch.bool, device="cuda")
    keep[300] = False
    assert torch.equal(p.w[0][keep], q.w[0][keep]) and torch.equal(p.w[1], q.w[1])
    m, v, m2, v2 = (torch.empty(p.n, device="cuda") for _ in range(4))
    B.a2sgd_adamw_read_state(p.plan, m, v)
    B.a2sgd_adamw_read_state(q.plan, m2, v2)
    off = torch.zeros(p.n, dtype=torch.bool, device="cuda")
    off[300 if bits == 32 else slice(256, 512)] = True
    assert not torch.isfinite(m[300]) and not torch.isfinite(v[300])
    assert torch.equal(m[~off], m2[~off]) and torch.equal(v[~off], v2[~off])


@pytest.mark.parametrize("bits", [32, 8])
def test_a_scale_that_is_not_finite_changes_nothing(bits):
    p = Problem([3000, 7], bits=bits, copy=torch.bfloat16)
    tensors = [t for t in (p.wbuf, p.cbuf, p.m, p.v, p.ms, p.vs) if t is not None]
    before = [t.clone() for t in tensors]
    p.g[1][3] = math.inf
    out = torch.zeros(2, device="cuda")
    B.a2sgd_adamw_grad_norm(p.plan, 1.0, out)
    assert math.isinf(out[0].item()) and math.isnan(out[1].item())
    B.a2sgd_adamw_step(p.plan, step=1, grad_scale=out[1:], **HYPER)
    for a, b in zip(tensors, before):
        assert torch.equal(a, b)


@pytest.mark.parametrize("numel", LISTS + [[3] * 700, [5_000_001]], ids=lambda x: "%dx%d" % (len(x), sum(x)))
@pytest.mark.parametrize("gtype,skew,gscale", [(torch.float32, 0, 1e-2), (torch.float32, 1, 1e25), (torch.float32, 0, 1e-30),
                                               (torch.bfloat16, 0, 1.0), (torch.float16, 5, 1.0)])
def test_grad_norm(numel, gtype, skew, gscale):
    """The squares' sum is exact to 2^-50 or so: what is left is one rounding to fp32 of each output."""
    p = Problem(numel, gtype, skew, gscale=gscale)
    norm = math.sqrt(sum((t.double() ** 2).sum().item() for t in p.g))
    out = torch.zeros(2, device="cuda")
    for limit in (norm * 0.25, norm * 4):
        limit = float(F32(limit))
        for _ in range(2):           # the second call finds the counter reset
            out.zero_()
            B.a2sgd_adamw_grad_norm(p.plan, limit, out)
            assert abs(out[0].item() - norm) <= 2 * U * norm
            assert abs(out[1].item() - min(1.0, limit / norm)) <= 3 * U


def test_same_bits_every_time_and_on_another_stream():
    outs = []
    side = torch.cuda.Stream()
    for k in range(3):
        p = Problem([70_001, 12, 100_000], bits=8, seed=11)
        out = torch.zeros(2, device="cuda")
        torch.cuda.synchronize()
        stream = side if k == 2 else None
        for step in (1, 2, 3):
            B.a2sgd_adamw_grad_norm(p.plan, 0.5, out, stream=stream)
            B.a2sgd_adamw_step(p.plan, step=step, grad_scale=out[1:], stream=stream, **HYPER)
        torch.cuda.synchronize()
        outs.append([t.clone() for t in (p.wbuf, p.m, p.v, p.ms, p.vs, out)])
    for other in outs[1:]:
        for a, b in zip(outs[0], other):
            assert torch.equal(a, b)


def test_refusals():
    p = Problem([1000])
    n = p.n
    ok = dict(step=1, **HYPER)
    for bad in (dict(lr=math.nan), dict(lr=-1.0), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0), dict(eps=1e-60),
                dict(weight_decay=-1.0)):
        with pytest.raises(B.A2SGDError) as e:
            B.a2sgd_adamw_step(p.plan, **{**ok, **bad})
        assert e.value.status == B.ERR_ARG
    with pytest.raises(ValueError):
        B.a2sgd_adamw_step(p.plan, **{**ok, "step": 0})
    for bad in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(B.A2SGDError):
            B.a2sgd_adamw_grad_norm(p.plan, bad, torch.zeros(2, device="cuda"))
    f = lambda k, dtype=torch.float32: torch.zeros(k, dtype=dtype, device="cuda")  # noqa: E731
    w, g = [f(1000)], [f(1000)]
    for args in ((w, [f(999)], f(n), f(n)), (w, g, f(n - 1), f(n)), (w, g, f(n), f(n), f(4), f(4)),
                 (w, g, f(n, torch.int8), f(n, torch.uint8)), (w, g, f(n, torch.int8), f(n, torch.int8), f(4), f(4)),
                 (w, g, f(n), f(n), None, None, [f(1000)]), ([f(1000).cpu()], g, f(n), f(n)), ([], [], f(n), f(n)),
                 ([f(1000, torch.float64)], g, f(n), f(n)), (w, [f(1000, torch.int32)], f(n), f(n)),
                 ([f(2000)[::2]], g, f(n), f(n))):
        with pytest.raises((ValueError, B.A2SGDError)):
            B.a2sgd_adamw_create(*args)
    with pytest.raises(B.A2SGDError) as e:               # the state is read 32 bytes at a time
        B.a2sgd_adamw_create(w, g, f(n + 1)[1:], f(n))
    assert e.value.status == B.ERR_ALIGN
    p.plan.destroy()
    with pytest.raises(RuntimeError):
        B.a2sgd_adamw_step(p.plan, **ok)
