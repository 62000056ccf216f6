"""Layer norm forward and backward through the binding, against the formulas in 64 bits and differences.

Tolerances.  u = 2^-24.  A sum of d values here is added in chains of at most 16 and trees above, 26 roundings
deep at most for the register forms; the long form chains d / 1024 values a thread: 16 + 26 at d <= 16384.  So a
sum of terms t is off by at most 42 u sum |t|.
Forward: the mean is off by e = 42 u mean|x|; xhat = (x - mean) rstd by (e + u |x|) rstd and by the relative error
of rstd, which second-order in e and 30 u; so |y - ref| <= |w| (2 (e + u|x|) rstd + 40 u |xhat|) + 2 u |y|,
plus half a unit in the last place of the output's type.
Backward (mean and rstd are inputs): c1 and c2 are off by 42 u of the means of |terms| and the roundings of xhat
(2 u max|xhat| amplification where x - mean cancels: (u |x| + u |mean|) rstd)."""
import numpy as np
import pytest
import torch

from paper_2006_07405_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF_ULP = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -25}


def _rows(values, dtype, pad, skew=0):
    r, c = values.shape
    buf = torch.full((r * (c + pad) + skew,), 9.0, device="cuda").to(dtype)
    out = buf[skew:].view(r, c + pad)[:, :c]
    out.copy_(values)
    return out, buf


def _problem(rows, d, dtype, param, pad=0, skew=0, offset=0.5, seed=0):
    gen = torch.Generator("cuda").manual_seed(seed)
    rnd = lambda *s: torch.empty(s, device="cuda").normal_(0, 1, generator=gen)  # noqa: E731
    x, _ = _rows(rnd(rows, d) + offset, dtype, pad, skew)
    dy, _ = _rows(rnd(rows, d), dtype, pad, skew)
    return x, dy, (1 + 0.2 * rnd(d)).to(param), (0.2 * rnd(d)).to(param)


def _forward64(x, w, b, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    rstd = ((x - mean).square().mean(1, keepdim=True) + eps).rsqrt()
    w = 1.0 if w is None else w.double()
    return (x - mean) * rstd * w + (0.0 if b is None else b.double()), mean, rstd


def _check_forward(x, w, b, y, mean, rstd, eps):
    ref, m, r = _forward64(x, w, b, eps)
    ax = x.double().abs()
    e = 42 * U * ax.mean(1, keepdim=True)
    aw = 1.0 if w is None else w.double().abs()
    xhat = (x.double() - m).abs() * r
    tol = aw * (2 * (e + U * ax) * r + 40 * U * xhat) + (2 * U + HALF_ULP[y.dtype]) * ref.abs() + TINY[y.dtype]
    tol = tol * (1 + HALF_ULP[y.dtype])
    assert torch.all((y.double() - ref).abs() <= tol)
    assert torch.all((mean.double() - m[:, 0]).abs() <= e[:, 0] + U * m[:, 0].abs() + 1e-44)
    # the variance: 45 u relative, and the square of the mean's error
    assert torch.all((rstd.double() - r[:, 0]).abs() <= r[:, 0] * (30 * U + (e * r).square()[:, 0]))


SHAPES = [(1, 1), (3, 7), (5, 8), (33, 31), (70, 64), (1, 256), (7, 257), (130, 777), (9, 1001), (64, 1600),
          (5000, 1600), (6000, 40), (2500, 72), (9000, 9), (3, 4096), (2, 4104), (1300, 4096), (3, 8192), (2, 8200), (3, 16384)]
TYPES = [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16),
         (torch.float16, torch.float32), (torch.float16, torch.float16)]


@pytest.mark.parametrize("rows,d", SHAPES)
@pytest.mark.parametrize("dtype,param", TYPES)
@pytest.mark.parametrize("pad,skew", [(0, 0), (5, 1)])
def test_forward(rows, d, dtype, param, pad, skew):
    x, _, w, b = _problem(rows, d, dtype, param, pad, skew)
    y, buf = _rows(torch.zeros(rows, d, device="cuda"), dtype, pad, skew)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.a2sgd_layer_norm_forward(x, w, b, y, mean, rstd, 1e-5)
    _check_forward(x, w, b, y, mean, rstd, 1e-5)
    if pad:
        assert torch.all(buf[skew:].view(rows, d + pad)[:, d:] == 9.0) and torch.all(buf[:skew] == 9.0)


@pytest.mark.parametrize("d", [64, 100, 1600, 8200])
def test_forward_with_a_large_mean_without_parameters_and_in_place(d):
    x, _, w, b = _problem(50, d, torch.float32, torch.float32, offset=1000.0)
    mean, rstd = torch.empty(50, device="cuda"), torch.empty(50, device="cuda")
    for w_, b_ in ((w, b), (None, b), (w, None), (None, None)):
        y = torch.empty_like(x)
        B.a2sgd_layer_norm_forward(x, w_, b_, y, mean, rstd, 1e-5)
        _check_forward(x, w_, b_, y, mean, rstd, 1e-5)
    z = x.clone()
    B.a2sgd_layer_norm_forward(z, None, None, z, None, None, 1e-5)
    assert torch.equal(z, y)


@pytest.mark.parametrize("d", [8, 100, 1600, 8200])
def test_constant_rows_and_rows_that_are_not_finite(d):
    """No spread: y is the bias (the mean of equal numbers may be off by roundings, times 1 / sqrt(eps)).  A row that
    holds NaN or infinity is NaN and alone in that."""
    x, _, w, b = _problem(6, d, torch.float32, torch.float32)
    x[1] = 4.0
    x[3, d // 2] = float("nan")
    x[4, 0] = float("inf")
    y = torch.empty_like(x)
    mean, rstd = torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    B.a2sgd_layer_norm_forward(x, w, b, y, mean, rstd, 1e-5)
    good = [0, 1, 2, 5]
    _check_forward(x[good], w, b, y[good], mean[good], rstd[good], 1e-5)
    assert torch.isnan(y[3]).all() and torch.isnan(y[4]).all()


def _check_backward(dy, x, w, mean, rstd, dx, dw, db):
    x64, g64 = x.double(), dy.double()
    m, r = mean.double()[:, None], rstd.double()[:, None]
    w64 = torch.ones(x.shape[1], device="cuda", dtype=torch.float64) if w is None else w.double()
    xhat = (x64 - m) * r
    ehat = U * (2 * (x64.abs() + m.abs()) * r + 2 * xhat.abs())         # x - mean and the product, rounded
    u = g64 * w64
    c1, c2 = u.mean(1, keepdim=True), (u * xhat).mean(1, keepdim=True)
    ref = r * (u - c1 - xhat * c2)
    e1 = 44 * U * u.abs().mean(1, keepdim=True)
    e2 = (44 * U * (u * xhat).abs() + u.abs() * ehat).mean(1, keepdim=True)
    tol = r * (4 * U * (u.abs() + c1.abs() + (xhat * c2).abs()) + e1 + xhat.abs() * e2 + ehat * c2.abs()) + HALF_ULP[dx.dtype] * ref.abs()
    assert torch.all((dx.double() - ref).abs() <= tol * (1 + HALF_ULP[dx.dtype]) + TINY[dx.dtype])
    # column sums: a chain over a CTA's rows, then its groups and the CTAs; rows / (CTAs) + 64 roundings at most
    depth = 64 + x.shape[0] / 100
    for got, terms, extra in ((dw, g64 * xhat, g64.abs() * ehat), (db, g64, 0 * g64)):
        tol = U * depth * terms.abs().sum(0) + extra.sum(0) + HALF_ULP[got.dtype] * terms.sum(0).abs()
        assert torch.all((got.double() - terms.sum(0)).abs() <= tol * (1 + HALF_ULP[got.dtype]) + TINY[got.dtype])


def _statistics(x, eps=1e-5):
    _, m, r = _forward64(x, None, None, eps)
    return m[:, 0].float().contiguous(), r[:, 0].float().contiguous()


@pytest.mark.parametrize("rows,d", SHAPES)
@pytest.mark.parametrize("dtype,param", TYPES)
@pytest.mark.parametrize("pad,skew", [(0, 0), (5, 1)])
def test_backward(rows, d, dtype, param, pad, skew):
    x, dy, w, _ = _problem(rows, d, dtype, param, pad, skew)
    mean, rstd = _statistics(x)
    dx, buf = _rows(torch.zeros(rows, d, device="cuda"), dtype, pad, skew)
    dw, db = torch.full((d,), 5.0, device="cuda").to(param), torch.full((d,), 5.0, device="cuda").to(param)
    work = torch.empty(B.a2sgd_layer_norm_workspace(rows, d), dtype=torch.uint8, device="cuda")
    B.a2sgd_layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db, work)
    _check_backward(dy, x, w, mean, rstd, dx, dw, db)
    if pad:
        assert torch.all(buf[skew:].view(rows, d + pad)[:, d:] == 9.0) and torch.all(buf[:skew] == 9.0)
    # parts of it give the same bits; dx may take the place of dy
    first = [t.clone() for t in (dx, dw, db)]
    dw.fill_(3)
    B.a2sgd_layer_norm_backward(dy, x, w, mean, rstd, None, dw, None, work)
    assert torch.equal(dw, first[1])
    B.a2sgd_layer_norm_backward(dy, x, w, mean, rstd, dy, None, db, work)
    assert torch.equal(dy, first[0]) and torch.equal(db, first[2])


@pytest.mark.parametrize("d", [24, 1001, 8200])
def test_backward_against_differences(d):
    """Central differences of f = sum(c y) in 64 bits; their own error is of the order h^2 = 1e-8 of the third derivative
    and eps / h = 1e-11, so 1e-5 relative to the gradient's scale covers it and the fp32 kernel."""
    rows = 3
    x, c, w, b = _problem(rows, d, torch.float32, torch.float32)
    mean, rstd = _statistics(x)
    dx, dw, db = torch.empty_like(x), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    work = torch.empty(B.a2sgd_layer_norm_workspace(rows, d), dtype=torch.uint8, device="cuda")
    B.a2sgd_layer_norm_backward(c, x, w, mean, rstd, dx, dw, db, work)
    f = lambda x_, w_, b_: (c.double() * _forward64(x_, w_, b_, 1e-5)[0]).sum().item()  # noqa: E731
    h = 1e-4
    rng = np.random.default_rng(0)
    x64, w64, b64 = x.double(), w.double(), b.double()
    for _ in range(12):
        i, j = int(rng.integers(rows)), int(rng.integers(d))
        for t, got, at in ((x64, dx, (i, j)), (w64, dw, (j,)), (b64, db, (j,))):
            keep = t[at].item()
            t[at] = keep + h
            up = f(x64, w64, b64)
            t[at] = keep - h
            down = f(x64, w64, b64)
            t[at] = keep
            assert abs((up - down) / (2 * h) - got[at].item()) <= 1e-5 * max(1.0, got.abs().max().item())


def test_no_rows_refusals_and_streams():
    f = lambda *s, dtype=torch.float32: torch.ones(s, dtype=dtype, device="cuda")  # noqa: E731
    d = 16
    work = torch.empty(B.a2sgd_layer_norm_workspace(0, d), dtype=torch.uint8, device="cuda")
    dw, db = f(d), f(d)
    B.a2sgd_layer_norm_forward(f(0, d), f(d), f(d), f(0, d), f(0), f(0))
    B.a2sgd_layer_norm_backward(f(0, d), f(0, d), f(d), f(0), f(0), f(0, d), dw, db, work)
    assert torch.all(dw == 0) and torch.all(db == 0)
    x = f(4, d)
    for call in (lambda: B.a2sgd_layer_norm_forward(x.cpu(), f(d), f(d), x, None, None),
                 lambda: B.a2sgd_layer_norm_forward(x, f(d + 1), f(d), x, None, None),
                 lambda: B.a2sgd_layer_norm_forward(x, f(d), f(d, dtype=torch.bfloat16), x, None, None),
                 lambda: B.a2sgd_layer_norm_forward(x, f(d, dtype=torch.bfloat16), None, x, None, None),
                 lambda: B.a2sgd_layer_norm_forward(x, f(d), f(d), f(4, d, dtype=torch.float16), None, None),
                 lambda: B.a2sgd_layer_norm_forward(x, f(d), f(d), f(5, d), None, None),
                 lambda: B.a2sgd_layer_norm_forward(x.double(), None, None, x.double(), None, None),
                 lambda: B.a2sgd_layer_norm_forward(f(4, 2 * d)[:, ::2], None, None, x, None, None),
                 lambda: B.a2sgd_layer_norm_forward(x[:1].expand(4, d), None, None, x, None, None),
                 lambda: B.a2sgd_layer_norm_forward(x, None, None, x, None, None, eps=-1.0),
                 lambda: B.a2sgd_layer_norm_forward(x, None, None, x, None, None, eps=float("nan")),
                 lambda: B.a2sgd_layer_norm_backward(x, x, f(d), f(4), f(4), x, f(d), f(d), None),
                 lambda: B.a2sgd_layer_norm_backward(x, x, f(d), f(4), f(4), x, f(d), f(d), work[:16]),
                 lambda: B.a2sgd_layer_norm_backward(x, x, f(d), f(3), f(4), x, f(d), f(d), work)):
        with pytest.raises((ValueError, B.A2SGDError)):
            call()
    x, dy, w, b = _problem(3000, 1600, torch.bfloat16, torch.float32)
    mean, rstd = _statistics(x)
    outs = []
    for stream in (None, torch.cuda.Stream()):
        torch.cuda.synchronize()
        y, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
        work = torch.empty(B.a2sgd_layer_norm_workspace(3000, 1600), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        B.a2sgd_layer_norm_forward(x, w, b, y, mean, rstd, stream=stream)
        B.a2sgd_layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db, work, stream=stream)
        torch.cuda.synchronize()
        outs.append((y, dx, dw, db))
    for a, b_ in zip(*outs):
        assert torch.equal(a, b_)
