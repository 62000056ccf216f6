"""The backward pass' parts of the first tokens' keys: the room for them without a GPU, and sequences of all lengths that have one, some or many."""
import ctypes
import math

import pytest
import torch

from attention_util import check, reference
from paper_2006_07405_b200 import binding as B


def backward_bytes(sequences, rows, q_heads, kv_heads, d, window, sinks, packed=True):
    s = B._AttentionShape(sequences, q_heads, kv_heads, d, rows, rows, None, None, window, sinks, B.BF16, 1.0)
    flags = B.ATTENTION_BACKWARD | B.ATTENTION_ALIGNED | (B.ATTENTION_PACKED_Q | B.ATTENTION_PACKED_K if packed else 0)
    return B.lib().a2sgd_window_attention_workspace(ctypes.addressof(s), flags)


@pytest.mark.parametrize("rows, q_heads, kv_heads, d, window, sinks", [(32768, 25, 25, 128, 64, 299), (131072, 32, 8, 128, 1024, 128), (262144, 32, 8, 128, 1024, 128)])
def test_room_grows_with_the_rows_not_with_the_sequences(rows, q_heads, kv_heads, d, window, sinks):
    rest = 2 * 4 * q_heads * rows + 4096
    group = q_heads // kv_heads
    each = max(32, ((127 + window + 63) // 64 + 1) * group)        # blocks of a part
    for sequences in (1, 2, 32, 128, 1024, 65535):
        # a part for each `each` blocks of 64 rows, two more for each sequence that can have several, with dk and dv of each first token
        several = min(sequences, rows // 193, rows * group // (64 * each) * 2)
        parts = rows * group // (64 * each) + 2 + 2 * several
        assert backward_bytes(sequences, rows, q_heads, kv_heads, d, window, sinks) <= rest + 20 * (several + 2) + 256 + parts * kv_heads * sinks * 2 * d * 4


def normal(gen, *shape, dtype=torch.bfloat16):
    return torch.empty(shape, device="cuda").normal_(generator=gen).to(dtype)


def run(q_lens, k_lens, q_packed, k_packed, hq, hkv, d, window, sinks, seed=0, dtype=torch.bfloat16, order=None):
    """Sequences in planes of their own, or behind one another with gaps (in another order than the ranges', with `order`); NaN where none is."""
    gen, n = torch.Generator("cuda").manual_seed(seed), len(q_lens)
    order = order or list(range(n))

    def place(lens, packed, gap):
        first, at = [0] * n, gap
        for b in order if packed else []:
            first[b], at = at, at + lens[b] + gap
        ranges = torch.tensor(list(zip(first, lens)), dtype=torch.int32, device="cuda")
        shape = (at,) if packed else (n, max(lens) + gap)
        return first, ranges, shape

    q_at, q_ranges, q_shape = place(q_lens, q_packed, 3)
    k_at, k_ranges, k_shape = place(k_lens, k_packed, 2)
    rows = lambda t, b, at, lens, packed: (t if packed else t[b])[at[b]:at[b] + lens[b]]  # noqa: E731

    def new(shape, h, at, lens, packed):
        t = torch.full((*shape, h, d), math.nan, dtype=dtype, device="cuda")
        for b in range(n):
            rows(t, b, at, lens, packed).copy_(normal(gen, lens[b], h, d, dtype=dtype))
        return t

    q, dout = (new(q_shape, hq, q_at, q_lens, q_packed) for _ in range(2))
    k, v = (new(k_shape, hkv, k_at, k_lens, k_packed) for _ in range(2))
    o, lse = torch.full_like(q, math.nan), torch.full((hq, q_shape[0]) if q_packed else (n, hq, q_shape[1]), math.nan, device="cuda")
    kw = dict(window=window, sinks=sinks, q_ranges=q_ranges, k_ranges=k_ranges)
    B.a2sgd_window_attention_forward(q, k, v, o, lse, workspace=torch.empty(B.a2sgd_window_attention_workspace(q, k, window, sinks, n), dtype=torch.uint8, device="cuda"), **kw)
    size = B.a2sgd_window_attention_workspace(q, k, window, sinks, n, backward=True)
    work = torch.full((size + 512,), 0xAB, dtype=torch.uint8, device="cuda")
    grads = [torch.full_like(t, math.nan) for t in (q, k, v)]
    B.a2sgd_window_attention_backward(dout, q, k, v, o, lse, *grads, workspace=work[:size], **kw)
    again = [torch.full_like(t, math.nan) for t in (q, k, v)]
    B.a2sgd_window_attention_backward(dout, q, k, v, o, lse, *again, workspace=work[:size], **kw)
    torch.cuda.synchronize()
    assert (work[size:] == 0xAB).all() and B.a2sgd_window_attention_status() == B.OK
    assert all(torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0)) for a, b in zip(grads, again))
    for t, at, lens, packed in ((grads[0], q_at, q_lens, q_packed), (grads[1], k_at, k_lens, k_packed), (grads[2], k_at, k_lens, k_packed)):
        outside = torch.ones(t.shape[:-2], dtype=torch.bool, device="cuda")
        for b in range(n):
            rows(outside, b, at, lens, packed).fill_(False)
        assert torch.isnan(t[outside]).all()
    for b in range(n):
        own = lse[:, q_at[b]:q_at[b] + q_lens[b]] if q_packed else lse[b, :, q_at[b]:q_at[b] + q_lens[b]]
        mine = [rows(t, b, q_at, q_lens, q_packed) for t in (q, dout, o, grads[0])]
        keys = [rows(t, b, k_at, k_lens, k_packed) for t in (k, v, grads[1], grads[2])]
        ref = reference(mine[0], keys[0], keys[1], window, sinks, d ** -0.5, mine[1], mine[2], own)
        for name, got in (("dq", mine[3]), ("dk", keys[2]), ("dv", keys[3])):
            check(f"{name} of {b}", got, *ref[name])


LONG = [2600, 1, 0, 140, 2300]


@pytest.mark.gpu
@pytest.mark.parametrize("q_packed, k_packed", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("sinks", [5, 140])
def test_several_sequences_and_key_heads(q_packed, k_packed, sinks):
    run(LONG, LONG, q_packed, k_packed, 4, 2, 64, 60, sinks, seed=sinks)
    run(LONG, [2650, 9, 30, 140, 2200], q_packed, k_packed, 3, 3, 72, 33, sinks, seed=sinks + 1, dtype=torch.float16)


@pytest.mark.gpu
def test_ranges_in_another_order():
    run([300, 2500, 0, 2100, 5], [300, 2500, 7, 2100, 5], True, True, 2, 1, 128, 60, 9, order=[3, 0, 4, 1, 2])


@pytest.mark.gpu
def test_planes_that_are_filled_in_part():
    run([2500, 2437], [2500, 2490], False, False, 4, 2, 64, 100, 130)


@pytest.mark.gpu
def test_more_sequences_than_a_list_is_made_of_at_once():
    """300 short ones, with long ones first, beyond the 256 that a CTA looks at together, and last."""
    lens = [i % 3 for i in range(300)]
    lens[0], lens[270], lens[299] = 2300, 2700, 2200
    run(lens, lens, True, True, 2, 1, 32, 40, 3)


@pytest.mark.gpu
def test_one_long_sequence_among_packed_rows():
    run([5000], [5000], True, True, 1, 1, 64, 70, 3)
    run([1, 5000, 1], [1, 5000, 1], True, True, 1, 1, 64, 70, 3)


@pytest.mark.gpu
@pytest.mark.parametrize("packed", [True, False])
def test_many_queries_and_no_keys(packed):
    run([200, 3, 130], [0, 0, 1], packed, packed, 2, 1, 64, 30, 2)


@pytest.mark.gpu
def test_captured_and_replayed_with_other_lengths():
    """The list of parts is the device's: a replay goes by the ranges as they are then."""
    gen, rows, window, sinks = torch.Generator("cuda").manual_seed(3), 5200, 60, 9
    q, dout = (normal(gen, rows, 4, 64) for _ in range(2))
    k, v = (normal(gen, rows, 2, 64) for _ in range(2))
    ranges = torch.tensor([[0, 200], [200, 5000], [5200, 0]], dtype=torch.int32, device="cuda")
    kw = dict(window=window, sinks=sinks, q_ranges=ranges, k_ranges=ranges)
    work = torch.empty(B.a2sgd_window_attention_workspace(q, k, window, sinks, 3, backward=True), dtype=torch.uint8, device="cuda")
    o, lse, grads = torch.zeros_like(q), torch.zeros((4, rows), device="cuda"), [torch.zeros_like(t) for t in (q, k, v)]

    def both(o, lse, grads, work):
        B.a2sgd_window_attention_forward(q, k, v, o, lse, workspace=work, **kw)
        B.a2sgd_window_attention_backward(dout, q, k, v, o, lse, *grads, workspace=work, **kw)

    both(o, lse, grads, work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(o, lse, grads, work)
    other = torch.empty_like(work)
    for lens in ([5000, 200, 0], [2500, 100, 2600], [1, 1, 5198], [1700, 1700, 1800]):
        first = [0, lens[0], lens[0] + lens[1]]
        ranges.copy_(torch.tensor(list(zip(first, lens)), dtype=torch.int32, device="cuda"))
        graph.replay()
        want = torch.zeros_like(q), torch.zeros((4, rows), device="cuda"), [torch.zeros_like(t) for t in (q, k, v)]
        both(*want, other)
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1]) and all(torch.equal(a, b) for a, b in zip(grads, want[2]))
    assert B.a2sgd_window_attention_status() == B.OK
