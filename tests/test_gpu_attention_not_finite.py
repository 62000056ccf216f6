"""Attention over tensors that are not finite in places: what sees such a place is not finite, as the formulas say, and nothing else is touched."""
import math

import pytest
import torch

from attention_util import reference, visible
from paper_2006_07405_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16}
BAD = [math.nan, math.inf, -math.inf]


def normal(gen, *shape, dtype):
    return torch.empty(shape, device="cuda").normal_(generator=gen).to(dtype)


def forward(q, k, v, window, sinks, **kw):
    o = torch.full_like(q, 7.0)
    lse = torch.full((q.shape[0], q.shape[2], q.shape[1]), 7.0, device="cuda")
    work = torch.empty(B.a2sgd_window_attention_workspace(q, k, window, sinks, q.shape[0]), dtype=torch.uint8, device="cuda")
    B.a2sgd_window_attention_forward(q, k, v, o, lse, window=window, sinks=sinks, workspace=work, **kw)
    assert B.a2sgd_window_attention_status() == B.OK
    return o, lse


def backward(dout, q, k, v, o, lse, window, sinks, **kw):
    grads = [torch.full_like(t, 7.0) for t in (q, k, v)]
    work = torch.empty(B.a2sgd_window_attention_workspace(q, k, window, sinks, q.shape[0], backward=True), dtype=torch.uint8, device="cuda")
    B.a2sgd_window_attention_backward(dout, q, k, v, o, lse, *grads, window=window, sinks=sinks, workspace=work, **kw)
    assert B.a2sgd_window_attention_status() == B.OK
    return grads


def formulas(q, k, v, window, sinks, dout=None, o=None, lse=None):
    """The definition in 64 bits for one sequence, hidden pairs left out of every sum."""
    lq, hq, d = q.shape
    lk, hkv = k.shape[:2]
    seen = visible(lq, lk, window, sinks, q.device)
    zero = torch.zeros((), dtype=torch.float64, device=q.device)
    out = {n: torch.zeros((r, h, d), dtype=torch.float64, device=q.device) for n, r, h in (("o", lq, hq), ("dq", lq, hq), ("dk", lk, hkv), ("dv", lk, hkv))}
    out["lse"] = torch.full((hq, lq), -math.inf, dtype=torch.float64, device=q.device)
    some, s3 = seen.any(1), seen[:, :, None]
    for h in range(hq):
        g = h // (hq // hkv)
        qq, kk, vv = q[:, h].double(), k[:, g].double(), v[:, g].double()
        # a product by itself for each pair: what one row holds does not reach another's
        x = (qq[:, None] * kk[None]).sum(-1) * d ** -0.5
        if dout is None:
            x = x.masked_fill(~seen, -math.inf)
            top = x.amax(1, keepdim=True)
            p = torch.where(seen, (x - top).exp(), zero)
            total = p.sum(1, keepdim=True)
            out["o"][:, h] = torch.where(some[:, None], torch.where(s3, p[:, :, None] * vv[None], zero).sum(1) / total, zero)
            out["lse"][h] = torch.where(some, (total.log() + top)[:, 0], out["lse"][h])
            continue
        dd, oo = dout[:, h].double(), o[:, h].double()
        p = torch.where(seen, (x - lse[h].double()[:, None]).exp(), zero)
        dp = (dd[:, None] * vv[None]).sum(-1)
        ds = torch.where(seen, p * (dp - (dd * oo).sum(1, keepdim=True)), zero)
        out["dq"][:, h] = d ** -0.5 * torch.where(s3, ds[:, :, None] * kk[None], zero).sum(1)
        out["dk"][:, g] += d ** -0.5 * torch.where(s3, ds[:, :, None] * qq[:, None], zero).sum(0)
        out["dv"][:, g] += torch.where(s3, p[:, :, None] * dd[:, None], zero).sum(0)
    return out


def compare(name, got, want, bound):
    """Finite where the formula is, and there within the bound; not finite elsewhere."""
    finite = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), finite), f"{name}: finite elsewhere, {(torch.isfinite(got) != finite).nonzero()[:8].tolist()}"
    off = ((got.double() - want).abs() - bound)[finite]
    assert off.numel() == 0 or off.max().item() <= 0.0, f"{name}: {off.max().item()} beyond its bound"


def check_forward(q, k, v, window, sinks, o, lse):
    want = formulas(q, k, v, window, sinks)
    plain = reference(*(t.nan_to_num(0.0, 0.0, 0.0) for t in (q, k, v)), window, sinks, q.shape[-1] ** -0.5)   # for its bounds
    compare("o", o, want["o"], plain["o"][1])
    empty = torch.isneginf(want["lse"])
    assert torch.equal(torch.isneginf(lse), empty), "lse: other rows are empty"
    compare("lse", lse.masked_fill(empty, 0.0), want["lse"].masked_fill(empty, 0.0), plain["lse"][1])


def check_backward(dout, q, k, v, o, lse, window, sinks, grads):
    want = formulas(q, k, v, window, sinks, dout, o, lse)
    clean = [t.nan_to_num(0.0, 0.0, 0.0) for t in (q, k, v, dout, o, lse)]
    # bounds: those of the finite parts; a pair's terms only shrink where something is put to 0, so the largest of each row is taken
    plain = reference(*clean[:3], window, sinks, q.shape[-1] ** -0.5, *clean[3:])
    for name, got in zip(("dq", "dk", "dv"), grads):
        compare(name, got, want[name], plain[name][1])


def places(n, d):
    """(row, column) of what is not finite: at the start, within a tile and a block, at their edges, and last."""
    return [(0, 3 % d), (70, d - 1), (n // 2, 0), (n - 1, d // 2)]


@pytest.mark.parametrize("which", ["q", "k", "v"])
@pytest.mark.parametrize("lq, lk", [(1, 300), (2, 40), (7, 300), (300, 300), (140, 60)])
@pytest.mark.parametrize("d, dtype", [(64, "bf16"), (128, "f16"), (72, "f16")])
def test_forward(which, lq, lk, d, dtype):
    """One row at a time in each of two heads: all of a row of q or k, one element of v."""
    gen = torch.Generator("cuda").manual_seed(lq + d)
    q0, k0, v0 = (normal(gen, 1, n, 2, d, dtype=DT[dtype]) for n in (lq, lk, lk))
    for i, bad in enumerate(BAD):
        for row, column in places(lq if which == "q" else lk, d):
            q, k, v = q0.clone(), k0.clone(), v0.clone()
            t = {"q": q, "k": k, "v": v}[which]
            row = min(row, t.shape[1] - 1)
            if which == "v":
                t[0, row, i % 2, column] = bad
            else:
                t[0, row, i % 2] = math.nan if which == "k" else bad
            for window, sinks in ((33, 2), (100, 75)):
                o, lse = forward(q, k, v, window, sinks)
                check_forward(q[0], k[0], v[0], window, sinks, o[0], lse[0])


def test_forward_several_at_once():
    """Opposite infinities in one column, next to NaN in others; rows that see none, one, or both."""
    gen = torch.Generator("cuda").manual_seed(3)
    for lq in (3, 400):
        q, k, v = (normal(gen, 1, n, 2, 64, dtype=torch.bfloat16) for n in (lq, 400, 400))
        v[0, 130, 0, 5], v[0, 135, 0, 5], v[0, 131, 1, 7], v[0, 399, 1, 9], v[0, 0, 1, 8] = math.inf, -math.inf, math.nan, math.inf, -math.inf
        for window, sinks in ((40, 1), (128, 0), (400, 0)):
            o, lse = forward(q, k, v, window, sinks)
            check_forward(q[0], k[0], v[0], window, sinks, o[0], lse[0])


@pytest.mark.parametrize("which", ["q", "k", "v", "dout"])
@pytest.mark.parametrize("lq, lk", [(300, 300), (140, 60), (3, 200)])
@pytest.mark.parametrize("hq, hkv, d, dtype", [(2, 2, 64, "bf16"), (3, 1, 128, "f16"), (4, 2, 40, "bf16")])
def test_backward(which, lq, lk, hq, hkv, d, dtype):
    gen = torch.Generator("cuda").manual_seed(lq + d)
    q0, k0, v0, g0 = (normal(gen, 1, n, h, d, dtype=DT[dtype]) for n, h in ((lq, hq), (lk, hkv), (lk, hkv), (lq, hq)))
    for i, bad in enumerate(BAD):
        for row, column in places(lk if which in "kv" else lq, d):
            q, k, v, dout = q0.clone(), k0.clone(), v0.clone(), g0.clone()
            t = {"q": q, "k": k, "v": v, "dout": dout}[which]
            row = min(row, t.shape[1] - 1)
            if which in ("v", "dout"):
                t[0, row, i % t.shape[2], column] = bad
            else:
                t[0, row, i % t.shape[2]] = math.nan
            for window, sinks in ((33, 2), (100, 75)):
                o, lse = forward(q, k, v, window, sinks)
                grads = backward(dout, q, k, v, o, lse, window, sinks)
                check_backward(dout[0], q[0], k[0], v[0], o[0], lse[0], window, sinks, [g[0] for g in grads])


def test_backward_of_many_queries_to_first_tokens():
    """The first tokens' passes in parts, with a gradient that is not finite in each of two of them, and a key that is not a number."""
    gen = torch.Generator("cuda").manual_seed(8)
    q, k, v, dout = (normal(gen, 1, 3000, 1, 32, dtype=torch.bfloat16) for _ in range(4))
    dout[0, 700, 0, 3], dout[0, 2500, 0, 9] = math.inf, math.nan
    o, lse = forward(q, k, v, 60, 5)
    grads = backward(dout, q, k, v, o, lse, 60, 5)
    check_backward(dout[0], q[0], k[0], v[0], o[0], lse[0], 60, 5, [g[0] for g in grads])


def test_one_infinite_element_of_a_key():
    """Its scores are infinite with either sign: a query of a lowest one goes on without the key, its gradient does not (0 times infinity)."""
    gen = torch.Generator("cuda").manual_seed(2)
    for lq in (4, 260):
        q, k, v, dout = (normal(gen, 1, n, 1, 64, dtype=torch.bfloat16) for n in (lq, 260, 260, lq))
        k[0, 250, 0, 11] = math.inf
        q[0, ::2, 0, 11], q[0, 1::2, 0, 11] = 1.0, -1.0
        o, lse = forward(q, k, v, 90, 1)
        seen = visible(lq, 260, 90, 1, "cuda")[:, 250]
        up = q[0, :, 0, 11] > 0
        assert torch.isnan(o[0, seen & up]).all() and torch.isfinite(o[0, ~(seen & up)]).all()
        grads = backward(dout, q, k, v, o, lse, 90, 1)
        want = formulas(q[0], k[0], v[0], 90, 1, dout[0], o[0], lse[0])
        for name, g in zip(("dq", "dk", "dv"), grads):
            assert torch.equal(torch.isfinite(g[0]), torch.isfinite(want[name])), name


def test_more_tiles_than_are_remembered():
    """Each tile of many has a place that is not finite, a CTA has more of them than its list: the same bits as with 0 there, elsewhere."""
    gen = torch.Generator("cuda").manual_seed(1)
    shape, d, c = (32, 2048, 64), 8, 3
    q, k, v, dout = (normal(gen, *shape, d, dtype=torch.bfloat16) for _ in range(4))
    bad = torch.arange(100, shape[1], 128, device="cuda")

    def run(value):
        v[:, bad, :, c] = value
        dout[:, bad, :, c] = 0.0
        o, lse = forward(q, k, v, 16, 0)
        dout[:, bad, :, c] = value
        # the gradients beside outputs that are finite: delta, and so dk and dq, is not where dout is not
        v[:, bad, :, c] = 0.0
        return o, lse, *backward(dout, q, k, v, o0, lse, 16, 0)

    v[:, bad, :, c] = 0.0
    o0, _ = forward(q, k, v, 16, 0)
    clean, got = run(0.0), run(math.nan)
    place = torch.arange(shape[1], device="cuda")
    sees = ((place[:, None] >= bad) & (place[:, None] < bad + 16)).any(1)       # queries that see a bad key
    seen = ((place[:, None] <= bad) & (place[:, None] > bad - 16)).any(1)       # keys that a bad query sees
    is_bad = (place[:, None] == bad).any(1)
    o, dq, dk, dv = torch.zeros_like(q, dtype=torch.bool), *(torch.zeros_like(q, dtype=torch.bool) for _ in range(3))
    o[:, sees, :, c], dv[:, seen, :, c], dq[:, is_bad], dk[:, seen] = True, True, True, True
    assert torch.equal(clean[1], got[1])
    for name, lost, a, b in (("o", o, clean[0], got[0]), ("dq", dq, clean[2], got[2]), ("dk", dk, clean[3], got[3]), ("dv", dv, clean[4], got[4])):
        assert torch.isnan(b[lost]).all() and torch.equal(a[~lost], b[~lost]), name


@pytest.mark.parametrize("bads", [[math.inf], [math.inf, -math.inf, math.nan]])
def test_more_blocks_of_a_pass_than_are_remembered(bads):
    """A first token's pass of 44 blocks (4 heads of 11) a part, a gradient that is not finite in each: 32 of them are listed."""
    gen = torch.Generator("cuda").manual_seed(6)
    n, d, h = 2100, 16, 4
    q, dout, k, v = (normal(gen, 1, n, x, d, dtype=torch.bfloat16) for x in (h, h, 1, 1))
    for i, row in enumerate(range(7, n, 50)):
        dout[0, row, :, 3] = bads[i % len(bads)]
    o, lse = forward(q, k, v, 500, 3)
    grads = backward(dout, q, k, v, o, lse, 500, 3)
    check_backward(dout[0], q[0], k[0], v[0], o[0], lse[0], 500, 3, [g[0] for g in grads])
    dout[0, 1500:, :, :] = math.nan
    grads = backward(dout, q, k, v, o, lse, 500, 3)
    check_backward(dout[0], q[0], k[0], v[0], o[0], lse[0], 500, 3, [g[0] for g in grads])


@pytest.mark.parametrize("d, wide", [(63, 64), (33, 40), (100, 104), (8, 9)])
def test_heads_inside_wider_ones(d, wide):
    """Rows whose last elements are not eight, and ones that are copied first; what lies behind a head is not a number and does not count."""
    gen = torch.Generator("cuda").manual_seed(d)
    new = lambda h: torch.full((1, 150, h, wide), math.nan, device="cuda", dtype=torch.bfloat16)[..., :d].copy_(normal(gen, 1, 150, h, d, dtype=torch.bfloat16))  # noqa: E731
    q, k, v, dout = new(4), new(2), new(2), new(4)
    v[0, 70, 0, d - 1], v[0, 149, 1, 0], dout[0, 90, 1, d - 1], k[0, 20, 1, d - 1] = math.inf, math.nan, -math.inf, math.nan
    o, lse = forward(q, k, v, 50, 2)
    check_forward(q[0], k[0], v[0], 50, 2, o[0], lse[0])
    grads = backward(dout, q, k, v, o, lse, 50, 2)
    check_backward(dout[0], q[0], k[0], v[0], o[0], lse[0], 50, 2, [g[0] for g in grads])
    o, lse = forward(q[:, :3], k, v, 50, 2)
    check_forward(q[0, :3], k[0], v[0], 50, 2, o[0], lse[0])
