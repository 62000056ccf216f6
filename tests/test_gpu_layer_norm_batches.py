"""Layer norm on batches large enough for the kernels that take many rows: the warp-a-row forward form, and several rows in
flight in CTAs that hold several groups.

The row counts go by the device's number of SMs and stay above the thresholds of the dispatch: forward, a warp a row takes
d = 257..2048 from 40 rows for each resident CTA of 128 threads on (16 of them at most); several rows are in flight from 8 rows
for each group of each SM on, a group being the threads of a row and a CTA holding 256 / group of them."""
import pytest
import torch

from paper_2006_07405_b200 import binding as B
from test_gpu_layer_norm import TYPES, _check_backward, _check_forward, _problem, _rows, _statistics

pytestmark = pytest.mark.gpu


def _sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def _many_rows(d):
    """Just over eight rows for each group of each SM, with a remainder."""
    need = -(-d // 8)
    tpr = 1 << (need - 1).bit_length() if need <= 32 else -(-need // 32) * 32
    groups = min(64, max(1, 256 // tpr if tpr <= 128 else 1))
    return _sms() * groups * 8 + 35


def _run(rows, d, dtype, param, pad=0, skew=0, backward=True, in_place=False):
    x, dy, w, b = _problem(rows, d, dtype, param, pad, skew, seed=rows + d)
    y, buf = _rows(torch.zeros(rows, d, device="cuda"), dtype, pad, skew)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.a2sgd_layer_norm_forward(x, w, b, y, mean, rstd, 1e-5)
    _check_forward(x, w, b, y, mean, rstd, 1e-5)
    if pad:
        assert torch.all(buf[skew:].view(rows, d + pad)[:, d:] == 9.0) and torch.all(buf[:skew] == 9.0)
    if in_place:
        z = x.clone()
        B.a2sgd_layer_norm_forward(z, w, b, z, mean, rstd, 1e-5)
        assert torch.equal(z, y)
    if not backward:
        return
    mean, rstd = _statistics(x)
    dx, buf = _rows(torch.zeros(rows, d, device="cuda"), dtype, pad, skew)
    dw, db = torch.full((d,), 5.0, device="cuda").to(param), torch.full((d,), 5.0, device="cuda").to(param)
    work = torch.empty(B.a2sgd_layer_norm_workspace(rows, d), dtype=torch.uint8, device="cuda")
    B.a2sgd_layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db, work)
    _check_backward(dy, x, w, mean, rstd, dx, dw, db)
    if pad:
        assert torch.all(buf[skew:].view(rows, d + pad)[:, d:] == 9.0) and torch.all(buf[:skew] == 9.0)
    if in_place:
        first = [t.clone() for t in (dx, dw, db)]
        B.a2sgd_layer_norm_backward(dy, x, w, mean, rstd, x, dw, db, work)
        for a, ref in zip((x, dw, db), first):
            assert torch.equal(a, ref)


@pytest.mark.parametrize("d", [264, 520, 776, 1024, 1200, 1600, 2048])
@pytest.mark.parametrize("dtype,param", TYPES)
def test_a_warp_a_row(d, dtype, param):
    """Every number of pieces a lane and every pair of types; the last piece whole (1024, 2048), and in part."""
    _run(_sms() * 16 * 40 + 7, d, dtype, param, pad=8 if d % 16 else 0, backward=False, in_place=dtype is torch.float32)


@pytest.mark.parametrize("d", [8, 24, 40, 72, 128, 256, 1024, 4096])
@pytest.mark.parametrize("dtype,param", TYPES)
def test_several_rows_in_flight(d, dtype, param):
    _run(_many_rows(d), d, dtype, param, in_place=True)


@pytest.mark.parametrize("d", [1, 9, 31, 40, 72, 255, 777, 1003, 4090])
@pytest.mark.parametrize("dtype,param", TYPES[:3])
def test_several_rows_in_flight_without_vector_accesses(d, dtype, param):
    _run(_many_rows(d), d, dtype, param, pad=5, skew=1)
