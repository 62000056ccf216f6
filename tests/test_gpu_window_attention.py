"""Windowed attention against its definition in 64 bits, through the binding."""
import math

import pytest
import torch

from attention_util import check, reference
from paper_2006_07405_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def heads(gen, *shape, dtype, pad=0, skew=0, std=1.0):
    """[..., heads, d] as a view of rows that are `pad` elements wider, `skew` elements into its buffer; NaN around."""
    *lead, h, d = shape
    rows = math.prod(lead)
    buf = torch.full((rows * (h * d + pad) + skew,), math.nan, dtype=dtype, device="cuda")
    view = buf[skew:].view(rows, h * d + pad)[:, :h * d]
    view.copy_(torch.empty((rows, h * d), device="cuda").normal_(0.0, std, generator=gen))
    strides, step = [], h * d + pad
    for n in reversed(lead):
        strides.insert(0, step)
        step *= n
    return buf.as_strided((*lead, h, d), (*strides, d, 1), skew)


def run(sequences, lq, lk, hq, hkv, d, window, sinks, dtype="bf16", pad=0, skew=0, q_lens=None, k_lens=None, packed=False, scale=None,
        backward=True, seed=0, std=1.0, aligned=False):
    """lq, lk: rows of a plane, used up to q_lens, k_lens; packed: sequences of these lengths with gaps of NaN between them."""
    gen, dt = torch.Generator("cuda").manual_seed(seed), DT[dtype]
    scale = d ** -0.5 if scale is None else scale
    q_lens, k_lens = q_lens or [lq] * sequences, k_lens or [lk] * sequences
    if packed:
        q_at, k_at, at_q, at_k = [], [], 3, 1
        for a, b in zip(q_lens, k_lens):
            q_at.append(at_q)
            k_at.append(at_k)
            at_q, at_k = at_q + a + 2, at_k + b + 5
        shape_q, shape_k = (at_q,), (at_k,)
    else:
        q_at, k_at = [0] * sequences, [0] * sequences
        shape_q, shape_k = (sequences, lq), (sequences, lk)
    kw = dict(dtype=dt, pad=pad, skew=skew, std=std)
    q, k, v = heads(gen, *shape_q, hq, d, **kw), heads(gen, *shape_k, hkv, d, **kw), heads(gen, *shape_k, hkv, d, **kw)
    o, dout = heads(gen, *shape_q, hq, d, **kw), heads(gen, *shape_q, hq, d, **kw)
    whole = not packed and q_lens == [lq] * sequences and k_lens == [lk] * sequences
    q_ranges = None if whole else torch.tensor(list(zip(q_at, q_lens)), dtype=torch.int32, device="cuda").view(-1, 2)
    k_ranges = None if whole else torch.tensor(list(zip(k_at, k_lens)), dtype=torch.int32, device="cuda").view(-1, 2)

    def cut(t, b, at, n):
        return t[at[b]:at[b] + n[b]] if packed else t[b, at[b]:at[b] + n[b]]

    def blank(t, at, n):   # what lies outside the sequences is NaN, and has to stay it
        keep = torch.zeros(t.shape[:-2], dtype=torch.bool, device="cuda")
        for b in range(sequences):
            (keep if packed else keep[b])[at[b]:at[b] + n[b]] = True
        t[~keep] = math.nan
        return keep

    for t in (q, o, dout):
        keep_q = blank(t, q_at, q_lens)
    for t in (k, v):
        keep_k = blank(t, k_at, k_lens)
    lse = torch.full((hq, shape_q[0]) if packed else (sequences, hq, lq), math.nan, device="cuda")
    common = dict(window=window, sinks=sinks, scale=scale, q_ranges=q_ranges, k_ranges=k_ranges)
    guard = 512

    def workspace(back):
        n = B.a2sgd_window_attention_workspace(q, k, window, sinks, sequences, backward=back, aligned=aligned)
        w = torch.full((n + guard,), 0xAB, dtype=torch.uint8, device="cuda")
        return w, w[:n]

    w, use = workspace(False)
    B.a2sgd_window_attention_forward(q, k, v, o, lse, workspace=use, **common)
    torch.cuda.synchronize()
    assert (w[use.numel():] == 0xAB).all()
    assert B.a2sgd_window_attention_status() == B.OK
    assert torch.isnan(o[~keep_q]).all()
    win = 1 << 31 if window is None else window
    for b in range(sequences):
        ref = reference(cut(q, b, q_at, q_lens), cut(k, b, k_at, k_lens), cut(v, b, k_at, k_lens), win, sinks, scale)
        check(f"o of {b}", cut(o, b, q_at, q_lens), *ref["o"])
        own = lse[:, q_at[b]:q_at[b] + q_lens[b]] if packed else lse[b, :, :q_lens[b]]
        check(f"lse of {b}", own, *ref["lse"])
    # without lse: the same bits
    again = torch.full_like(o, math.nan)
    B.a2sgd_window_attention_forward(q, k, v, again, None, workspace=use, **common)
    assert torch.equal(again[keep_q], o[keep_q])
    if not backward:
        return
    dq, dk, dv = torch.full_like(q, math.nan), torch.full_like(k, math.nan), torch.full_like(v, math.nan)
    w, use = workspace(True)
    B.a2sgd_window_attention_backward(dout, q, k, v, o, lse, dq, dk, dv, workspace=use, **common)
    torch.cuda.synchronize()
    assert (w[use.numel():] == 0xAB).all()
    assert B.a2sgd_window_attention_status() == B.OK
    assert torch.isnan(dq[~keep_q]).all() and torch.isnan(dk[~keep_k]).all() and torch.isnan(dv[~keep_k]).all()
    for b in range(sequences):
        own = lse[:, q_at[b]:q_at[b] + q_lens[b]] if packed else lse[b, :, :q_lens[b]]
        ref = reference(cut(q, b, q_at, q_lens), cut(k, b, k_at, k_lens), cut(v, b, k_at, k_lens), win, sinks, scale,
                        cut(dout, b, q_at, q_lens), cut(o, b, q_at, q_lens), own)
        check(f"dq of {b}", cut(dq, b, q_at, q_lens), *ref["dq"])
        check(f"dk of {b}", cut(dk, b, k_at, k_lens), *ref["dk"])
        check(f"dv of {b}", cut(dv, b, k_at, k_lens), *ref["dv"])
    # one gradient at a time: the same bits, nothing else written
    for which in range(3):
        outs = [torch.full_like(t, math.nan) if i == which else None for i, t in enumerate((q, k, v))]
        B.a2sgd_window_attention_backward(dout, q, k, v, o, lse, *outs, workspace=use, **common)
        keep, want = (keep_q, dq) if which == 0 else (keep_k, (dk, dv)[which - 1])
        assert torch.equal(outs[which][keep], want[keep])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq, hkv, d", [(2, 2, 64), (6, 2, 128), (3, 1, 80), (2, 1, 40), (1, 1, 8)])
def test_whole_sequences(dtype, hq, hkv, d):
    run(2, 300, 300, hq, hkv, d, 97, 5, dtype=dtype)


@pytest.mark.parametrize("window, sinks", [(1, 0), (1, 1), (2, 300), (63, 0), (64, 64), (65, 65), (128, 127), (129, 200), (500, 3), (None, 0), (None, 9)])
@pytest.mark.parametrize("d", [64, 128])
def test_windows_and_first_tokens(window, sinks, d):
    run(1, 500, 500, 2, 1, d, window, sinks, seed=3)


@pytest.mark.parametrize("lq, lk", [(1, 1), (1, 2), (2, 1), (5, 0), (3, 1000), (127, 129), (128, 128), (129, 127), (64, 700), (300, 40), (257, 513)])
def test_lengths(lq, lk):
    """More queries than keys: the first ones see nothing."""
    run(2, lq, lk, 4, 2, 64, 100, 3, seed=lq)


@pytest.mark.parametrize("d", [1, 7, 16, 24, 63, 65, 72, 100, 127])
def test_head_dims(d):
    run(1, 200, 200, 2, 2, d, 70, 2, dtype="f16", seed=d)


@pytest.mark.parametrize("pad, skew", [(8, 0), (0, 8), (3, 0), (0, 1), (5, 3)])
def test_strides_and_addresses(pad, skew):
    run(2, 150, 150, 3, 1, 64, 50, 4, pad=pad, skew=skew)
    run(2, 150, 150, 3, 1, 128, 50, 4, pad=pad, skew=skew, dtype="f16")


@pytest.mark.parametrize("d", [64, 128])
def test_packed_sequences(d):
    lens = [1, 130, 0, 256, 77, 400]
    run(6, 0, 0, 4, 2, d, 90, 6, q_lens=lens, k_lens=lens, packed=True)
    run(6, 0, 0, 4, 2, d, 90, 6, q_lens=lens, k_lens=[5, 0, 9, 300, 77, 128], packed=True, dtype="f16")


def test_padded_sequences():
    run(4, 260, 260, 4, 4, 64, 120, 8, q_lens=[260, 1, 0, 129], k_lens=[260, 200, 30, 64])


@pytest.mark.parametrize("lq", [1, 2, 4, 9])
@pytest.mark.parametrize("hq, hkv, d", [(4, 4, 64), (8, 1, 128), (12, 2, 96), (32, 1, 64)])
def test_few_queries_over_a_cache(lq, hq, hkv, d):
    run(3, lq, 700, hq, hkv, d, 256, 7, q_lens=[lq] * 3, k_lens=[700, 1, 333], backward=False)
    run(2, lq, 2500, hq, hkv, d, None, 0, backward=False, dtype="f16")
    run(1, lq, 1100, hq, hkv, d, 64, 513, backward=False)


def test_few_queries_backward():
    run(2, 3, 300, 4, 2, 64, 100, 130, q_lens=[3, 2], k_lens=[300, 9])


def test_long_sequence():
    """Many tiles of first tokens' queries: the sum for the first keys is long."""
    run(1, 4100, 4100, 1, 1, 64, 200, 5)
    run(1, 2100, 2100, 2, 1, 128, 130, 140, dtype="f16")


def test_large_scores():
    """Scores far apart: the running maximum moves by more than the exponential's range."""
    run(1, 300, 300, 2, 2, 64, 150, 4, std=6.0)


def test_scores_that_grow():
    """A maximum that rises from tile to tile, by steps below and above what is put off."""
    gen = torch.Generator("cuda").manual_seed(5)
    n, d = 1024, 64
    q = torch.ones((1, n, 1, d), device="cuda", dtype=torch.bfloat16)
    k = (torch.arange(n, device="cuda")[None, :, None, None] // 64 * 0.75).expand(1, n, 1, d).to(torch.bfloat16).contiguous()
    v = torch.empty((1, n, 1, d), device="cuda").normal_(generator=gen).to(torch.bfloat16)
    for sign in (1.0, -1.0):
        o, lse = torch.empty_like(q), torch.empty((1, 1, n), device="cuda")
        B.a2sgd_window_attention_forward(q, (k * sign).contiguous(), v, o, lse, window=700, sinks=2, workspace=torch.empty(
            B.a2sgd_window_attention_workspace(q, k, 700, 2, 1), dtype=torch.uint8, device="cuda"))
        ref = reference(q[0], (k * sign)[0], v[0], 700, 2, d ** -0.5)
        check("o", o[0], *ref["o"])
        check("lse", lse[0], *ref["lse"])


def test_keys_outside_the_ranges_do_not_matter():
    """Infinities where no sequence is (the other tests have NaN there)."""
    gen = torch.Generator("cuda").manual_seed(1)
    q, k, v = (heads(gen, 1, 200, 2, 64, dtype=torch.bfloat16) for _ in range(3))
    ranges = torch.tensor([[0, 130]], dtype=torch.int32, device="cuda")
    outs = []
    for fill in (0.0, math.inf, -math.inf):
        for t in (k, v, q):
            t[:, 130:] = fill
        o = torch.zeros_like(q)
        w = torch.empty(B.a2sgd_window_attention_workspace(q, k, 60, 2, 1), dtype=torch.uint8, device="cuda")
        B.a2sgd_window_attention_forward(q, k, v, o, window=60, sinks=2, q_ranges=ranges, k_ranges=ranges, workspace=w)
        outs.append(o)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2]) and torch.isfinite(outs[0]).all()


def test_head_major_and_broadcast_layouts():
    """[sequence, head, row] in memory, and one key head's row for every sequence."""
    gen = torch.Generator("cuda").manual_seed(2)
    new = lambda *s: torch.empty(s, device="cuda").normal_(generator=gen).to(torch.bfloat16)  # noqa: E731
    q, k, v = new(3, 4, 170, 64).transpose(1, 2), new(1, 2, 170, 64).transpose(1, 2).expand(3, -1, -1, -1), new(3, 170, 1, 64).expand(-1, -1, 2, -1)
    o, lse = torch.empty_like(q), torch.empty((3, 4, 170), device="cuda")
    w = torch.empty(B.a2sgd_window_attention_workspace(q, k, 90, 3, 3, backward=True), dtype=torch.uint8, device="cuda")
    B.a2sgd_window_attention_forward(q, k, v, o, lse, window=90, sinks=3, workspace=w)
    dout = torch.randn(q.shape, device="cuda", generator=gen).to(torch.bfloat16)
    dq, dk, dv = torch.empty_like(q), torch.empty((3, 170, 2, 64), device="cuda", dtype=q.dtype), torch.empty((3, 170, 2, 64), device="cuda", dtype=q.dtype)
    B.a2sgd_window_attention_backward(dout, q, k, v, o, lse, dq, dk, dv, window=90, sinks=3, workspace=w)
    for b in range(3):
        ref = reference(q[b], k[b], v[b], 90, 3, 0.125)
        check("o", o[b], *ref["o"])
        ref = reference(q[b], k[b], v[b], 90, 3, 0.125, dout[b], o[b], lse[b])
        for n, t in (("dq", dq), ("dk", dk), ("dv", dv)):
            check(n, t[b], *ref[n])


def test_ranges_beyond_the_plane_are_clipped():
    gen = torch.Generator("cuda").manual_seed(2)
    q, k, v = (heads(gen, 2, 100, 1, 64, dtype=torch.float16) for _ in range(3))
    w = torch.empty(B.a2sgd_window_attention_workspace(q, k, 40, 0, 2), dtype=torch.uint8, device="cuda")
    outs = []
    for rows in ([[0, 100], [50, 50]], [[-7, 100000], [50, 2147483647]]):
        r = torch.tensor(rows, dtype=torch.int32, device="cuda")
        o = torch.zeros_like(q)
        B.a2sgd_window_attention_forward(q, k, v, o, window=40, q_ranges=r, k_ranges=r, workspace=w)
        outs.append(o)
    assert torch.equal(*outs)


def test_gradients_by_differences():
    """Directional derivatives of a loss that is linear in o, by central differences in 64 bits, against the kernel's gradients."""
    gen = torch.Generator("cuda").manual_seed(11)
    n, d = 90, 32
    q, k, v, dout = (torch.empty((1, n, 2, d), device="cuda").normal_(generator=gen).to(torch.float16) for _ in range(4))
    o, lse = torch.empty_like(q), torch.empty((1, 2, n), device="cuda")
    w = torch.empty(B.a2sgd_window_attention_workspace(q, k, 33, 2, 1, backward=True), dtype=torch.uint8, device="cuda")
    grads = [torch.empty_like(q) for _ in range(3)]
    B.a2sgd_window_attention_forward(q, k, v, o, lse, window=33, sinks=2, workspace=w)
    B.a2sgd_window_attention_backward(dout, q, k, v, o, lse, *grads, window=33, sinks=2, workspace=w)

    def loss(parts):
        total = 0.0
        for h in range(2):
            x = (parts[0][0, :, h] @ parts[1][0, :, h].T) * d ** -0.5
            i, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
            x = x.masked_fill(~((j <= i) & ((j > i - 33) | (j < 2))), -math.inf)
            total += ((torch.softmax(x, 1) @ parts[2][0, :, h]) * dout[0, :, h].double()).sum()
        return total.item()

    base = [t.double() for t in (q, k, v)]
    for i in range(3):
        step = torch.empty(q.shape, device="cuda", dtype=torch.float64).normal_(generator=gen)
        plus, minus = list(base), list(base)
        plus[i], minus[i] = base[i] + 1e-5 * step, base[i] - 1e-5 * step
        want = (loss(plus) - loss(minus)) / 2e-5
        # the kernel's gradients carry half a step of float16 twice, in n * 2 * d random terms: 6 deviations of their sum
        slack = 6 * 2 * 2.0 ** -11 * (grads[i].double() * step).norm().item() + 1e-6 * abs(want)
        assert abs((grads[i].double() * step).sum().item() - want) <= slack


def test_twice_the_same_bits_and_captured():
    gen = torch.Generator("cuda").manual_seed(4)
    q, k, v, dout = (torch.empty((2, 333, 4, 64), device="cuda").normal_(generator=gen).to(torch.bfloat16) for _ in range(4))
    w = torch.empty(B.a2sgd_window_attention_workspace(q, k, 100, 4, 2, backward=True), dtype=torch.uint8, device="cuda")

    def both(o, lse, grads):
        B.a2sgd_window_attention_forward(q, k, v, o, lse, window=100, sinks=4, workspace=w)
        B.a2sgd_window_attention_backward(dout, q, k, v, o, lse, *grads, window=100, sinks=4, workspace=w)

    outs = [(torch.empty_like(q), torch.empty((2, 4, 333), device="cuda"), [torch.empty_like(q) for _ in range(3)]) for _ in range(3)]
    both(*outs[0])
    both(*outs[1])
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        both(*outs[2])
    graph.replay()
    torch.cuda.synchronize()
    for other in outs[1:]:
        assert torch.equal(outs[0][0], other[0]) and torch.equal(outs[0][1], other[1])
        assert all(torch.equal(a, b) for a, b in zip(outs[0][2], other[2]))


def test_no_sequences_and_no_rows():
    q = torch.empty((0, 5, 2, 64), dtype=torch.bfloat16, device="cuda")
    B.a2sgd_window_attention_forward(q, q, q, torch.empty_like(q), window=3)
    q, k = torch.empty((2, 0, 2, 64), dtype=torch.bfloat16, device="cuda"), torch.randn((2, 5, 2, 64), device="cuda").to(torch.bfloat16)
    B.a2sgd_window_attention_forward(q, k, k, torch.empty_like(q), window=3)
    dk, dv = torch.full_like(k, math.nan), torch.full_like(k, math.nan)
    w = torch.empty(B.a2sgd_window_attention_workspace(q, k, 3, 0, 2, backward=True), dtype=torch.uint8, device="cuda")
    B.a2sgd_window_attention_backward(q, q, k, k, q, torch.empty((2, 2, 0), device="cuda"), None, dk, dv, window=3, workspace=w)
    assert not dk.any() and not dv.any()


def test_refusals():
    q = torch.zeros((2, 8, 4, 64), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((2, 8, 2, 64), dtype=torch.bfloat16, device="cuda")
    o = torch.empty_like(q)
    go = lambda **kw: B.a2sgd_window_attention_forward(**{**dict(q=q, k=k, v=k, o=o, window=4), **kw})  # noqa: E731
    go()
    for bad in (dict(q=q.float()), dict(k=k.half()), dict(v=k[:1]), dict(o=o[:, :4]), dict(window=0), dict(sinks=-1), dict(q=q[0]),
                dict(q_ranges=torch.zeros((3, 2), dtype=torch.int32, device="cuda")), dict(k_ranges=torch.zeros((2, 2), device="cuda")),
                dict(lse=torch.empty((2, 8, 4), device="cuda")), dict(k=k.cpu(), v=k.cpu()), dict(k=k.transpose(2, 3), v=k.transpose(2, 3)),
                dict(k=k[..., :32], v=k[..., :32])):
        with pytest.raises(ValueError):
            go(**bad)
    for bad, status in ((dict(scale=0.0), B.ERR_ARG), (dict(scale=math.inf), B.ERR_ARG), (dict(scale=-1.0), B.ERR_ARG),
                        (dict(o=o[:1].expand(2, -1, -1, -1)), B.ERR_ARG), (dict(o=o[:, :, :1].expand(-1, -1, 4, -1)), B.ERR_ARG),
                        (dict(q=q[:, :, :3], o=o[:, :, :3]), B.ERR_ARG)):
        with pytest.raises(B.A2SGDError) as e:
            go(**bad)
        assert e.value.status == status
    wide = torch.zeros((1, 4, 1, 136), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B.A2SGDError) as e:
        B.a2sgd_window_attention_forward(wide, wide, wide, torch.empty_like(wide))
    assert e.value.status == B.ERR_TOO_LARGE
    # not aligned, and no room to copy to
    odd = torch.zeros((2, 8, 4, 65), dtype=torch.bfloat16, device="cuda")[..., 1:]
    lse = torch.zeros((2, 4, 8), device="cuda")
    with pytest.raises(B.A2SGDError) as e:
        B.a2sgd_window_attention_backward(odd, q, k, k, o, lse, torch.empty_like(q), None, None, window=4)
    assert e.value.status == B.ERR_ARG
