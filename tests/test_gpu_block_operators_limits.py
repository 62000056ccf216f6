"""Attention, rotary positions and the residual connection at the ends of what they take: offsets beyond 2^31 elements, heads inside wider
ones, other streams, many short sequences."""
import math

import pytest
import torch

from attention_util import check, reference
from paper_2006_07405_b200 import binding as B

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def far_rows(gen, rows, heads, d, dtype):
    """Rows 2^24 elements apart: the last ones lie beyond 2^31 elements.  What is between is never written."""
    buf = torch.empty(((rows - 1) << 24) + heads * d, dtype=dtype, device="cuda")
    view = buf.as_strided((rows, heads, d), (1 << 24, d, 1))
    view.copy_(torch.empty((rows, heads, d), device="cuda").normal_(generator=gen))
    return view


def attention(q, k, v, dout, window, sinks, sequences=1, **kw):
    o = torch.empty_strided(q.shape, q.stride(), dtype=q.dtype, device="cuda") if q.stride(-3) < 1 << 24 else torch.empty(q.shape, dtype=q.dtype, device="cuda")
    lse = torch.empty((q.shape[1], q.shape[0]) if q.dim() == 3 else (q.shape[0], q.shape[2], q.shape[1]), device="cuda")
    work = torch.empty(B.a2sgd_window_attention_workspace(q, k, window, sinks, sequences, backward=True), dtype=torch.uint8, device="cuda")
    B.a2sgd_window_attention_forward(q, k, v, o, lse, window=window, sinks=sinks, workspace=work, **kw)
    grads = [torch.empty(t.shape, dtype=t.dtype, device="cuda") for t in (q, k, v)]
    if dout is not None:
        B.a2sgd_window_attention_backward(dout, q, k, v, o, lse, *grads, window=window, sinks=sinks, workspace=work, **kw)
    assert B.a2sgd_window_attention_status() == B.OK
    return o, lse, grads


def check_all(q, k, v, dout, window, sinks, o, lse, grads):
    scale = q.shape[-1] ** -0.5
    ref = reference(q, k, v, window, sinks, scale)
    check("o", o, *ref["o"])
    check("lse", lse, *ref["lse"])
    if dout is None:
        return
    ref = reference(q, k, v, window, sinks, scale, dout, o, lse)
    for name, g in zip(("dq", "dk", "dv"), grads):
        check(name, g, *ref[name])


@pytest.mark.parametrize("d", [64, 128])
def test_attention_beyond_two_to_the_31(d):
    gen = torch.Generator("cuda").manual_seed(1)
    k, v = far_rows(gen, 140, 1, d, BF16), far_rows(gen, 140, 1, d, BF16)
    q, dout = (torch.empty((140, 2, d), device="cuda").normal_(generator=gen).to(BF16) for _ in range(2))
    o, lse, grads = attention(q[None], k[None], v[None], dout[None], 70, 3)
    check_all(q, k, v, dout, 70, 3, o[0], lse[0], [g[0] for g in grads])
    o, lse, _ = attention(q[None, :3], k[None], v[None], None, 70, 3)         # few queries
    check_all(q[:3], k, v, None, 70, 3, o[0], lse[0], None)
    del k, v
    q, dout = far_rows(gen, 140, 1, d, BF16), far_rows(gen, 140, 1, d, BF16)
    k, v = (torch.empty((140, 1, d), device="cuda").normal_(generator=gen).to(BF16) for _ in range(2))
    o, lse, grads = attention(q[None], k[None], v[None], dout[None], 70, 3)
    check_all(q, k, v, dout, 70, 3, o[0], lse[0], [g[0] for g in grads])


@pytest.mark.parametrize("d, wide", [(63, 64), (40, 48), (100, 104), (33, 35)])
def test_attention_heads_inside_wider_ones(d, wide):
    """Strides that are aligned although head_dim is not a multiple of 8, and some that are not."""
    gen = torch.Generator("cuda").manual_seed(d)
    new = lambda h: torch.full((1, 150, h, wide), math.nan, device="cuda", dtype=BF16)[..., :d].copy_(torch.empty((1, 150, h, d), device="cuda").normal_(generator=gen))  # noqa: E731
    q, k, v, dout = new(4), new(2), new(2), new(4)
    o, lse, grads = attention(q, k, v, dout, 50, 2)
    check_all(q[0], k[0], v[0], dout[0], 50, 2, o[0], lse[0], [g[0] for g in grads])
    o, lse, _ = attention(q[:, :2], k, v, None, 50, 2)
    check_all(q[0, :2], k[0], v[0], None, 50, 2, o[0], lse[0], None)


def test_attention_many_short_sequences():
    """More sequences than a warp looks through at once, some of them empty."""
    gen = torch.Generator("cuda").manual_seed(7)
    lens = [(i * 7) % 11 for i in range(150)]
    first, at = [], 0
    for n in lens:
        first.append(at)
        at += n
    q, k, v, dout = (torch.empty((at, 2, 64), device="cuda").normal_(generator=gen).to(BF16) for _ in range(4))
    ranges = torch.tensor(list(zip(first, lens)), dtype=torch.int32, device="cuda")
    o, lse, grads = attention(q, k, v, dout, 4, 1, sequences=150, q_ranges=ranges, k_ranges=ranges)
    for a, n in zip(first, lens):
        cut = slice(a, a + n)
        check_all(q[cut], k[cut], v[cut], dout[cut], 4, 1, o[cut], lse[:, cut], [g[cut] for g in grads])


def test_attention_one_head_to_many():
    gen = torch.Generator("cuda").manual_seed(9)
    q, dout = (torch.empty((1, 200, 33, 64), device="cuda").normal_(generator=gen).to(BF16) for _ in range(2))
    k, v = (torch.empty((1, 200, 1, 64), device="cuda").normal_(generator=gen).to(BF16) for _ in range(2))
    o, lse, grads = attention(q, k, v, dout, 60, 5)
    check_all(q[0], k[0], v[0], dout[0], 60, 5, o[0], lse[0], [g[0] for g in grads])


def test_few_queries_shared_out_and_not():
    """One short and one long cache: no shares, shares within a cluster, and shares that a second launch joins; and without room for them."""
    gen = torch.Generator("cuda").manual_seed(4)
    for keys, d in ((100, 64), (3000, 64), (20000, 64), (9000, 128)):
        q = torch.empty((1, 2, 2, d), device="cuda").normal_(generator=gen).to(BF16)
        k, v = (torch.empty((1, keys, 1, d), device="cuda").normal_(generator=gen).to(BF16) for _ in range(2))
        work = torch.empty(B.a2sgd_window_attention_workspace(q, k, None, 0, 1, aligned=True), dtype=torch.uint8, device="cuda")
        for w in (work, None):
            o, lse = torch.empty_like(q), torch.empty((1, 2, 2), device="cuda")
            B.a2sgd_window_attention_forward(q, k, v, o, lse, workspace=w)
            check_all(q[0], k[0], v[0], None, 1 << 30, 0, o[0], lse[0], None)


@pytest.mark.parametrize("d, window, sinks", [(64, 1 << 30, 0), (128, 20000, 40), (72, 17000, 2)])
def test_shares_of_caches_of_all_lengths(d, window, sinks):
    """Two tiles of rows a key head, caches of 30000, 5 and no keys in one call: most shares of the short ones see nothing."""
    gen = torch.Generator("cuda").manual_seed(6)
    q = torch.empty((3, 2, 24, d), device="cuda").normal_(generator=gen).to(BF16)
    k, v = (torch.empty((3, 30000, 2, d), device="cuda").normal_(generator=gen).to(BF16) for _ in range(2))
    ranges = torch.tensor([[0, 30000], [7, 5], [0, 0]], dtype=torch.int32, device="cuda")
    work = torch.empty(B.a2sgd_window_attention_workspace(q, k, window, sinks, 3, aligned=True), dtype=torch.uint8, device="cuda")
    o, lse = torch.empty_like(q), torch.empty((3, 24, 2), device="cuda")
    again = torch.empty_like(q)
    B.a2sgd_window_attention_forward(q, k, v, o, lse, window=window, sinks=sinks, k_ranges=ranges, workspace=work)
    B.a2sgd_window_attention_forward(q, k, v, again, None, window=window, sinks=sinks, k_ranges=ranges, workspace=work)
    assert torch.equal(o, again)
    for b, (first, count) in enumerate(ranges.tolist()):
        check_all(q[b], k[b, first:first + count], v[b, first:first + count], None, window, sinks, o[b], lse[b], None)


def test_on_another_stream_and_side_by_side():
    """Two calls at once on two streams, with a workspace each."""
    gen = torch.Generator("cuda").manual_seed(5)
    sets = [[torch.empty((2, 500, 4, 64), device="cuda").normal_(generator=gen).to(BF16) for _ in range(4)] for _ in range(2)]
    want = [attention(*s, 100, 3, sequences=2) for s in sets]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for s, stream in zip(sets, streams):
        q, k, v, dout = s
        o, lse, grads = torch.empty_like(q), torch.empty((2, 4, 500), device="cuda"), [torch.empty_like(q) for _ in range(3)]
        work = torch.empty(B.a2sgd_window_attention_workspace(q, k, 100, 3, 2, backward=True), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        got.append((o, lse, grads, work))
    for (q, k, v, dout), stream, (o, lse, grads, work) in zip(sets, streams, got):
        B.a2sgd_window_attention_forward(q, k, v, o, lse, window=100, sinks=3, workspace=work, stream=stream)
        B.a2sgd_window_attention_backward(dout, q, k, v, o, lse, *grads, window=100, sinks=3, workspace=work, stream=stream)
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert torch.equal(w[0], g[0]) and torch.equal(w[1], g[1]) and all(torch.equal(a, b) for a, b in zip(w[2], g[2]))


@pytest.mark.parametrize("d", [1600, 4096, 8192])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_residual_without_the_first_norm_again_and_again(kind, d):
    """One norm a row: its warps' sums have two places, in turn, as a warp may be a row ahead of another."""
    gen = torch.Generator("cuda").manual_seed(9)
    x, y, dz, du = (torch.empty((6007, d), device="cuda").normal_(generator=gen).to(BF16) for _ in range(4))
    first = None
    for _ in range(20):
        z, u, dx, dy = (torch.empty_like(x) for _ in range(4))
        mean, rstd = torch.empty(6007, device="cuda"), torch.empty(6007, device="cuda")
        B.a2sgd_residual_norm_forward(x, y, z, u, kind, post=False, pre_mean=mean, pre_rstd=rstd)
        B.a2sgd_residual_norm_backward(dz, du, y, z, dx, dy, kind, post=False, pre_mean=mean, pre_rstd=rstd)
        out = [z, u, dx, dy, mean, rstd]
        first = first or out
        assert all(torch.equal(a, b) for a, b in zip(first, out))
    # 64-bit: the statistics are of z before its rounding; d products and sums in fp32, the root's and the quotient's rounding
    zz = x.double() + y.double()
    m = zz.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(zz[:, :1])
    r = ((zz - m).square().mean(1) + 1e-5).rsqrt()
    assert ((rstd.double() - r).abs() <= (d + 8) * 2.0 ** -24 * r).all()


def test_rotary_beyond_two_to_the_31():
    gen = torch.Generator("cuda").manual_seed(1)
    q = far_rows(gen, 140, 2, 64, BF16)
    near = q.clone()
    pos = torch.arange(140, dtype=torch.int32, device="cuda")[None].contiguous()
    out, want = torch.empty((140, 2, 64), dtype=BF16, device="cuda"), torch.empty((140, 2, 64), dtype=BF16, device="cuda")
    B.a2sgd_rotary(q, None, out, None, pos, [32])
    B.a2sgd_rotary(near, None, want, None, pos, [32])
    assert torch.equal(out, want)
    B.a2sgd_rotary(q, None, q, None, pos, [32])
    assert torch.equal(q, want)


def test_residual_beyond_two_to_the_31():
    gen = torch.Generator("cuda").manual_seed(1)
    y = far_rows(gen, 140, 1, 64, BF16)[:, 0]
    x = torch.empty((140, 64), device="cuda").normal_(generator=gen)
    outs = []
    for rows in (y, y.clone()):
        z, u, r1, r2 = torch.empty_like(x), torch.empty((140, 64), dtype=BF16, device="cuda"), torch.empty(140, device="cuda"), torch.empty(140, device="cuda")
        B.a2sgd_residual_norm_forward(x, rows, z, u, post_rstd=r1, pre_rstd=r2)
        dx, dy = torch.empty_like(x), torch.empty((140, 64), dtype=BF16, device="cuda")
        B.a2sgd_residual_norm_backward(None, u, rows, z, dx, dy, post_rstd=r1, pre_rstd=r2)
        outs.append((z, u, dx, dy))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
