"""Layer norm on rows and batches long enough for the order of the sums to show, and for 32-bit places to run out.

A thread adds at most 512 terms to one running sum; a row's or a column's runs of 512 are added up in turn, then the
threads' or CTAs' sums, with the sizes here under 100 roundings more: 512 + runs + 100 of at most u of the sum of
magnitudes.  One chain of n equal numbers drifts by 1939 u of its sum for 1.0681161 and n = 7812, by 4089 u for
1.9697274 and n = 16384 (added up in single precision on the host)."""
import pytest
import torch

from paper_2006_07405_b200 import binding as B
from test_gpu_layer_norm import HALF_ULP, TINY, U, _check_forward

pytestmark = pytest.mark.gpu


def _sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def _bound(runs):
    return (512 + runs + 100) * U


@pytest.mark.parametrize("d", [4096, 8200])
def test_column_sums_of_many_rows(d):
    """Equal rows: dw = rows * xhat with xhat = (1 - 0) * rstd, db = rows.  A CTA a row and SM at d = 4096, 64 slices of the
    rows at d = 8200: some 7800 rows each."""
    c = 1.0681161
    rows = 7812 * (_sms() if d == 4096 else 64)
    x = torch.ones((rows, d), dtype=torch.bfloat16, device="cuda")
    mean, rstd = torch.zeros(rows, device="cuda"), torch.full((rows,), c, device="cuda")
    dw, db = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
    work = torch.empty(B.a2sgd_layer_norm_workspace(rows, d), dtype=torch.uint8, device="cuda")
    B.a2sgd_layer_norm_backward(x, x, None, mean, rstd, None, dw, db, work)
    ref = rows * rstd[0].double().item()
    assert torch.all((dw.double() - ref).abs() <= _bound(7812 / 512 + 1) * ref)
    assert torch.all(db == rows)                    # whole numbers below 2^24
    # and the rows' gradients are as for a few of them
    g = 0.75
    mean, rstd = torch.zeros(rows, device="cuda"), torch.linspace(0.5, 2.0, rows, device="cuda")
    dy = torch.full_like(x, g)
    dy[:, ::2] = -g
    B.a2sgd_layer_norm_backward(dy, x, None, mean, rstd, dy, dw, db, work)
    want = torch.where(torch.arange(d, device="cuda") % 2 == 0, -g, g)
    for at in (0, 1, rows // 2, rows // 3 * 2 + 1, rows - 2, rows - 1):   # both means are zero
        ref = want.double() * rstd[at].double()
        assert torch.all((dy[at].double() - ref).abs() <= (HALF_ULP[torch.bfloat16] + 4 * U) * ref.abs())
    s = rstd.double().sum().item() * g
    assert torch.all((dw.double().abs() - s).abs() <= (_bound(7812 / 512 + 1) + 4 * U) * s)


@pytest.mark.parametrize("d", [8, 9, 72, 777, 1600])
def test_several_runs_of_rows_in_several_groups(d):
    """More than 512 rows for each group of four CTAs an SM, so that the second launch adds to the first one's sums: with and without
    vector accesses, one group a CTA (1600) and up to 64 (8), in place and beside it.  The groups' and CTAs' sums take at most 64 + 19 + 32
    roundings more; a term's own three are 4 u of (|x| + |mean|) rstd |dy|."""
    need = -(-d // 8)
    tpr = 1 << (need - 1).bit_length() if need <= 32 else -(-need // 32) * 32
    groups = min(64, max(1, 256 // tpr if tpr <= 128 else 1))
    rows = 512 * _sms() * 4 * groups + 12_345
    gen = torch.Generator("cuda").manual_seed(d)
    x = torch.empty((rows, d), dtype=torch.bfloat16, device="cuda").normal_(0.5, 1.0, generator=gen)
    dy = torch.empty((rows, d), dtype=torch.bfloat16, device="cuda").normal_(0.25, 1.0, generator=gen)
    mean = torch.empty(rows, device="cuda").normal_(0.5, 0.1, generator=gen)
    rstd = torch.empty(rows, device="cuda").uniform_(0.5, 1.5, generator=gen)
    w = torch.linspace(0.5, 1.5, d, device="cuda")
    dw, db = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
    work = torch.empty(B.a2sgd_layer_norm_workspace(rows, d), dtype=torch.uint8, device="cuda")
    dx = torch.empty_like(x)
    B.a2sgd_layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db, work)
    want_w, want_b, mag_w, mag_b, own = (torch.zeros(d, dtype=torch.float64, device="cuda") for _ in range(5))
    step = max(1, (1 << 26) // d)
    for lo in range(0, rows, step):
        p = slice(lo, min(rows, lo + step))
        g, m, r = dy[p].double(), mean[p].double()[:, None], rstd[p].double()[:, None]
        xhat = (x[p].double() - m) * r
        want_w += (g * xhat).sum(0)
        mag_w += (g * xhat).abs().sum(0)
        own += ((x[p].double().abs() + m.abs()) * r * g.abs()).sum(0)
        want_b += g.sum(0)
        mag_b += g.abs().sum(0)
    bound = (512 + 4 + 64 + 19 + 32) * U
    assert torch.all((dw.double() - want_w).abs() <= bound * mag_w + 4 * U * own)
    assert torch.all((db.double() - want_b).abs() <= bound * mag_b)
    # rows of the later launches are as a few rows alone
    for lo in (0, rows // 2, rows - 100):
        p, few = slice(lo, lo + 100), torch.empty((100, d), dtype=torch.bfloat16, device="cuda")
        B.a2sgd_layer_norm_backward(dy[p], x[p], w, mean[p], rstd[p], few, None, None)
        err = (dx[p].double() - few.double()).abs()        # the same sums in another order, then half a unit each
        assert torch.all(err <= 2.02 * HALF_ULP[torch.bfloat16] * few.double().abs() + 1e-4)
    first = dx.clone()
    B.a2sgd_layer_norm_backward(dy, x, w, mean, rstd, dy, dw, None, work)
    assert torch.equal(dy, first)


def test_sums_of_long_rows():
    d, c = 1 << 24, 1.9697274
    runs = d / 1024 / 512
    x = torch.full((1, d), c, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    B.a2sgd_layer_norm_forward(x, None, None, y, mean, rstd, 1e-5)
    ref = x[0, 0].double().item()
    assert abs(mean.double().item() - ref) <= _bound(runs) * ref
    # the variance: columns of +e and -e, whose mean is zero by symmetry; rstd has half its relative error
    e = c ** 0.5
    x.fill_(e)
    x[0, ::2] = -e
    B.a2sgd_layer_norm_forward(x, None, None, y, mean, rstd, 0.0)
    assert mean.item() == 0.0
    ref = 1.0 / abs(x[0, 0].double().item())
    assert abs(rstd.double().item() - ref) <= (0.5 * _bound(runs) + 4 * U) * ref
    # the two means of the backward pass: dy = c, xhat = 1, so dx = c - c - c
    dy, dx = torch.full_like(x, c), torch.empty_like(x)
    x.fill_(1.0)
    mean.zero_()
    rstd.fill_(1.0)
    B.a2sgd_layer_norm_backward(dy, x, None, mean, rstd, dx, None, None)
    ref = dy[0, 0].double().item()
    assert torch.all((dx.double() + ref).abs() <= (2 * _bound(runs) + 8 * U) * ref)


def test_more_than_2_31_elements():
    rows, d = 1_400_003, 1600
    gen = torch.Generator("cuda").manual_seed(0)
    x = torch.empty((rows, d), dtype=torch.bfloat16, device="cuda").normal_(0.5, 1.0, generator=gen)
    w, b = torch.linspace(0.5, 1.5, d, device="cuda"), torch.linspace(-1, 1, d, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.a2sgd_layer_norm_forward(x, w, b, y, mean, rstd, 1e-5)
    cross = (1 << 31) // d
    for lo in (0, cross - 20, rows - 40):
        part = slice(lo, lo + 40)
        _check_forward(x[part], w, b, y[part], mean[part], rstd[part], 1e-5)
    dx, dw, db = torch.empty_like(x), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    work = torch.empty(B.a2sgd_layer_norm_workspace(rows, d), dtype=torch.uint8, device="cuda")
    B.a2sgd_layer_norm_backward(y, x, w, mean, rstd, dx, dw, db, work)
    for lo in (0, cross - 20, rows - 40):
        p = slice(lo, lo + 40)
        few = torch.empty((40, d), dtype=torch.bfloat16, device="cuda")
        B.a2sgd_layer_norm_backward(y[p], x[p], w, mean[p], rstd[p], few, None, None)
        err = (dx[p].double() - few.double()).abs()        # the same sums in another order, then half a unit each
        assert torch.all(err <= 2 * HALF_ULP[torch.bfloat16] * few.double().abs() * 1.01 + 1e-3 * TINY[torch.float16])
    want_w, want_b, mag_w, mag_b = (torch.zeros(d, dtype=torch.float64, device="cuda") for _ in range(4))
    for lo in range(0, rows, 100_000):
        p = slice(lo, min(rows, lo + 100_000))
        g, xhat = y[p].double(), (x[p].double() - mean[p].double()[:, None]) * rstd[p].double()[:, None]
        want_w += (g * xhat).sum(0)
        mag_w += (g * xhat).abs().sum(0) + g.abs().sum(0)
        want_b += g.sum(0)
        mag_b += g.abs().sum(0)
    assert torch.all((dw.double() - want_w).abs() <= _bound(20) * mag_w)
    assert torch.all((db.double() - want_b).abs() <= _bound(20) * mag_b)
