"""The residual norm's column sums over batches long enough for the order of the additions to show, and their workspace.

A thread adds at most 512 rows to one running sum, at most 512 of these to the next, and then those, the CTAs' sums after them: with the sizes here
512 + 512 + 40 + 100 roundings at most, each of at most u of the sum of magnitudes.  One chain of 7812 numbers 1.0681161 drifts by 1939 u of its sum."""
import math

import pytest
import torch

from paper_2006_07405_b200 import binding as B
from test_gpu_residual_norm import both

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BOUND = (512 + 512 + 40 + 100) * U
C = 1.0681161


def _sums(rows, d, gate_rows, **kw):
    """Rows of ones throughout (the output's weight is 0, so that t is dz): sums of `rows` equal terms each."""
    one = torch.ones((rows, d), dtype=torch.bfloat16, device="cuda")
    rstd = torch.full((rows,), C, device="cuda")
    groups = -(-rows // gate_rows)
    new = lambda n: torch.full((n,), math.nan, device="cuda")  # noqa: E731
    names = ("dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias")
    sums = {n: new(d) for n in names}
    dgate = new(groups * d).view(groups, d)
    work = torch.empty(B.a2sgd_residual_norm_workspace(rows, d, gate_rows), dtype=torch.uint8, device="cuda")
    B.a2sgd_residual_norm_backward(one, one, one, one, None, None, "rms", post_weight=torch.ones(d, device="cuda"), gate=torch.ones((groups, d), device="cuda"),
                                   gate_rows=gate_rows, pre_weight=torch.zeros(d, device="cuda"), post_rstd=rstd, pre_rstd=rstd, dgate=dgate, workspace=work, **sums)
    return sums, dgate, rstd[0].double().item()


@pytest.mark.parametrize("d, ctas", [(64, 1024), (1600, 444), (4104, 148), (63, 1024)])
def test_many_rows(d, ctas):
    rows = ctas * 7812
    sums, dgate, c = _sums(rows, d, rows)
    for name, want in (("dpost_weight", rows * c), ("dpre_weight", rows * c), ("dpost_bias", rows), ("dpre_bias", rows)):
        off = (sums[name].double() - want).abs().max().item()
        assert off <= BOUND * want, (name, off / want / U)
    assert ((dgate.double() - rows * c).abs() <= BOUND * rows * c).all()


@pytest.mark.parametrize("d, gate_rows", [(64, 3), (72, 700), (4104, 1), (64, 5000)])
def test_many_gates(d, gate_rows):
    """More gates than one chain takes; gates of more rows than one, whole ones and ones that CTAs share."""
    rows = (1024 if d < 100 else 148) * 1953
    sums, dgate, c = _sums(rows, d, gate_rows)
    for name, want in (("dpost_weight", rows * c), ("dpre_weight", rows * c), ("dpost_bias", rows), ("dpre_bias", rows)):
        off = (sums[name].double() - want).abs().max().item()
        assert off <= BOUND * want, (name, off / want / U)
    last = rows - (dgate.shape[0] - 1) * gate_rows
    want = torch.full((dgate.shape[0], 1), float(gate_rows), dtype=torch.float64, device="cuda") * c
    want[-1] = last * c
    assert ((dgate.double() - want).abs() <= BOUND * want).all()


@pytest.mark.parametrize("rows, d, gate_rows, kind", [(150 * 1100, 96, 700, "layer"), (1200 * 520, 40, 1030, "rms"), (700, 5000, 300, "layer"), (3000, 8192, 0, "rms"),
                                                      (2900, 6001, 7, "layer")])
def test_runs_that_end_inside_gates(rows, d, gate_rows, kind):
    both(rows=rows, d=d, kind=kind, gate_rows=gate_rows, residual="f32")


@pytest.mark.parametrize("d", [1600, 4096, 8192])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_one_norm_a_row_with_the_sums_again_and_again(kind, d):
    gen = torch.Generator("cuda").manual_seed(2)
    x, y, dz, du = (torch.empty((6007, d), device="cuda").normal_(generator=gen).to(torch.bfloat16) for _ in range(4))
    z, u, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(6007, device="cuda"), torch.empty(6007, device="cuda")
    B.a2sgd_residual_norm_forward(x, y, z, u, kind, post=False, pre_mean=mean, pre_rstd=rstd)
    gate = torch.ones((2, d), device="cuda")
    work = torch.empty(B.a2sgd_residual_norm_workspace(6007, d, 4000), dtype=torch.uint8, device="cuda")
    first = None
    for _ in range(10):
        out = [torch.full_like(x, math.nan), torch.full_like(x, math.nan), *(torch.full((d,), math.nan, device="cuda") for _ in range(2)), torch.full((2, d), math.nan, device="cuda")]
        B.a2sgd_residual_norm_backward(dz, du, y, z, out[0], out[1], kind, post=False, gate=gate, gate_rows=4000, pre_mean=mean, pre_rstd=rstd,
                                       dpre_weight=out[2], dpre_bias=out[3], dgate=out[4], workspace=work)
        first = first or out
        assert all(torch.equal(a, b) for a, b in zip(first, out))
    hat = (z.double() - (mean.double()[:, None] if kind == "layer" else 0.0)) * rstd.double()[:, None]
    terms = du.double() * hat
    # fp32: a term's own roundings and at most 512 + 600 additions
    assert ((out[2].double() - terms.sum(0)).abs() <= (1112 + 8) * U * (du.double().abs() * (hat.abs() + (mean.double().abs() * rstd.double())[:, None])).sum(0)).all()
    assert ((out[3].double() - du.double().sum(0)).abs() <= 1112 * U * du.double().abs().sum(0)).all()


@pytest.mark.parametrize("d, ctas", [(8192, 1), (5000, 2), (2048, 4)])
def test_room_is_what_the_device_uses(d, ctas):
    """Four sums and, with a gate, two more of each CTA; a CTA an SM at d = 8192 (196 KB of shared memory each), few at other widths.  Several gates, or many
    rows: four sums more."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert B.a2sgd_residual_norm_workspace(65536, d) <= sms * ctas * 4 * d * 4
    assert B.a2sgd_residual_norm_workspace(65536, d, 1000) <= sms * ctas * 10 * d * 4
    assert B.a2sgd_residual_norm_workspace(1 << 24, d) <= sms * ctas * 8 * d * 4
    assert B.a2sgd_residual_norm_workspace(3, d) == 3 * 4 * d * 4 and B.a2sgd_residual_norm_workspace(0, d) == 0


def test_too_little_room_is_refused():
    one = torch.ones((2000, 64), dtype=torch.bfloat16, device="cuda")
    rstd, sums = torch.ones(2000, device="cuda"), torch.empty(64, device="cuda")
    n = B.a2sgd_residual_norm_workspace(2000, 64)
    work = torch.empty(n, dtype=torch.uint8, device="cuda")
    for size in (4 * 64 * 4, n // 4 // 256 * 256):
        with pytest.raises(B.A2SGDError) as e:
            B.a2sgd_residual_norm_backward(one, one, one, one, None, None, "rms", post=False, pre_rstd=rstd, dpre_weight=sums, workspace=work[:size])
        assert e.value.status == B.ERR_ARG
    B.a2sgd_residual_norm_backward(one, one, one, one, None, None, "rms", post=False, pre_rstd=rstd, dpre_weight=sums, workspace=work)
    assert (sums == 2000).all()
