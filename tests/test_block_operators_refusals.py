"""What the attention's, the rotary positions' and the residual connection's entry points refuse, through the C ABI, before anything is launched: no
GPU is needed, and no address here is ever read."""
import ctypes
import math

import pytest

from paper_2006_07405_b200 import binding as B

FAKE = 1 << 40      # an address that nothing reads


def heads(p=FAKE, seq=1 << 16, row=256, head=64):
    return (ctypes.c_int64 * 4)(p, seq, row, head)


def rows(p=FAKE, stride=64):
    return (ctypes.c_int64 * 2)(p, stride)


def at(x):
    return ctypes.addressof(x) if x is not None else None


def shape(**kw):
    s = dict(sequences=2, q_heads=4, kv_heads=2, head_dim=64, q_rows=8, k_rows=8, q_ranges=None, k_ranges=None, window=4, sinks=0, dtype=B.BF16,
             scale=0.125)
    s.update(kw)
    return B._AttentionShape(*s.values())


def forward(s, q=None, k=None, v=None, o=None, lse=None, workspace=None, bytes_=0):
    t = [heads() if x is None else x for x in (q, k, v, o)]
    return B.lib().a2sgd_window_attention_forward(at(s), *(at(x) if x != 0 else None for x in t), lse, workspace, bytes_, 0, None)


@pytest.mark.parametrize("bad", [dict(dtype=B.F32), dict(dtype=7), dict(q_heads=3), dict(q_heads=0), dict(kv_heads=0), dict(head_dim=0), dict(window=0),
                                 dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf)])
def test_attention_shapes(bad):
    assert forward(shape(**bad)) == B.ERR_ARG


@pytest.mark.parametrize("bad", [dict(head_dim=129), dict(q_rows=1 << 30), dict(k_rows=1 << 30), dict(sequences=70000), dict(q_heads=65536, kv_heads=1)])
def test_attention_sizes(bad):
    assert forward(shape(**bad)) == B.ERR_TOO_LARGE


def test_attention_tensors():
    s = shape()
    assert forward(s, q=0) == B.ERR_ARG and forward(s, v=heads(p=0)) == B.ERR_ARG and forward(s, o=0) == B.ERR_ARG
    assert forward(s, k=heads(row=-8)) == B.ERR_ARG
    assert forward(s, q=heads(p=FAKE + 1)) == B.ERR_ALIGN
    assert forward(s, lse=FAKE + 2) == B.ERR_ALIGN
    assert forward(s, workspace=FAKE + 64, bytes_=1 << 20) == B.ERR_ALIGN
    # packed queries and an output that is not, and the other way round
    assert forward(shape(q_ranges=FAKE), q=heads(seq=0)) == B.ERR_ARG and forward(shape(q_ranges=FAKE), o=heads(seq=0)) == B.ERR_ARG
    # outputs whose elements share a place
    assert forward(s, o=heads(seq=0)) == B.ERR_ARG and forward(s, o=heads(row=0)) == B.ERR_ARG and forward(s, o=heads(head=0)) == B.ERR_ARG
    assert B.lib().a2sgd_window_attention_forward(None, at(heads()), at(heads()), at(heads()), at(heads()), None, None, 0, 0, None) == B.ERR_ARG
    assert forward(shape(sequences=0), q=0) == B.OK and forward(shape(q_rows=0), q=0) == B.OK


def test_attention_backward():
    t = heads()
    go = lambda s, args, lse=FAKE, ws=FAKE, n=1 << 30: B.lib().a2sgd_window_attention_backward(  # noqa: E731
        at(s), *(at(x) for x in args[:5]), lse, *(at(x) for x in args[5:]), ws, n, 0, None)
    assert go(shape(), [t, t, t, t, None, t, t, t]) == B.ERR_ARG
    assert go(shape(), [t] * 8, lse=None) == B.ERR_ARG
    assert go(shape(), [t] * 5 + [heads(head=0), None, None]) == B.ERR_ARG
    assert go(shape(), [t] * 5 + [None, heads(row=0), None]) == B.ERR_ARG
    assert go(shape(k_ranges=FAKE), [t, t, heads(seq=0), heads(seq=0), t, None, t, None]) == B.ERR_ARG
    assert go(shape(k_ranges=FAKE), [t] * 7 + [heads(seq=0)]) == B.ERR_ARG
    assert go(shape(q_ranges=FAKE), [t, heads(seq=0), t, t, t, t, None, None]) == B.ERR_ARG
    assert go(shape(), [t] * 8, ws=FAKE + 8) == B.ERR_ALIGN
    assert go(shape(window=0), [t] * 8) == B.ERR_ARG


def test_attention_workspace():
    size = lambda s, flags: B.lib().a2sgd_window_attention_workspace(at(s), flags)  # noqa: E731
    long = dict(q_rows=4096, k_rows=4096)
    assert size(shape(**long), B.ATTENTION_ALIGNED) == 0
    assert size(shape(**long), 0) == 2 * 4096 * (4 + 2 * 2) * 64 * 2
    back = size(shape(**long), B.ATTENTION_ALIGNED | B.ATTENTION_BACKWARD)
    assert back == 2 * 2 * 4 * 4096 * 4 + 256     # lse and delta; counters
    # the first tokens' keys' shares: by key, part, dk and dv
    assert size(shape(sinks=5, window=64, **long), B.ATTENTION_ALIGNED | B.ATTENTION_BACKWARD) > back
    packed = B.ATTENTION_PACKED_Q | B.ATTENTION_PACKED_K
    assert size(shape(**long), packed) == 4096 * (4 + 2 * 2) * 64 * 2
    assert size(shape(head_dim=200), 0) == 0 and B.lib().a2sgd_window_attention_workspace(None, 0) == 0


def rotary(q=None, k=None, qo=None, ko=None, positions=FAKE, sections=(16, 16), base=10000.0, flags=0, tokens=4, hq=2, hk=1, d=64, dtype=B.F32, axes=None):
    t = [heads() if x is None else x for x in (q, k, qo, ko)]
    sec = (ctypes.c_uint32 * max(1, len(sections)))(*sections)
    return B.lib().a2sgd_rotary(*(at(x) if x != 0 else None for x in t), positions, len(sections) if axes is None else axes, at(sec), base, flags,
                                tokens, hq, hk, d, dtype, 0, None)


def test_rotary():
    for bad in (dict(dtype=9), dict(sections=(0, 4)), dict(sections=(20, 13)), dict(sections=()), dict(sections=(1,) * 5), dict(base=0.0), dict(base=-2.0),
                dict(base=math.inf), dict(flags=8), dict(d=0, sections=(1,)), dict(hq=0), dict(positions=None), dict(q=0), dict(ko=0), dict(qo=heads(row=0)),
                dict(q=heads(head=-1))):
        assert rotary(**bad) == B.ERR_ARG, bad
    for bad in (dict(d=513), dict(tokens=1 << 31), dict(hq=70000), dict(hk=70000)):
        assert rotary(**bad) == B.ERR_TOO_LARGE, bad
    assert rotary(positions=FAKE + 2) == B.ERR_ALIGN and rotary(q=heads(p=FAKE + 2)) == B.ERR_ALIGN
    assert rotary(tokens=0, q=0, k=0, qo=0, ko=0, positions=None) == B.OK


def residual(**kw):
    s = dict(rows=4, gate_rows=0, d=64, flags=B.RESIDUAL_RMS, dtype=B.BF16, residual_dtype=B.F32, param_dtype=B.F32, reserved=0, alpha=1.0, eps=1e-5,
             post_weight=None, post_bias=None, gate=None, pre_weight=None, pre_bias=None, post_mean=None, post_rstd=None, pre_mean=None, pre_rstd=None)
    s.update(kw)
    return B._ResidualShape(*s.values())


def test_residual_forward():
    go = lambda s, x=None, y=None, z=None, u=None: B.lib().a2sgd_residual_norm_forward(  # noqa: E731
        at(s), *(at(rows()) if t is None else (at(t) if t != 0 else None) for t in (x, y, z, u)), 0, None)
    for bad in (dict(dtype=5), dict(residual_dtype=B.F16), dict(param_dtype=B.F16), dict(d=0), dict(flags=4), dict(alpha=math.nan), dict(gate=FAKE), dict(eps=-1.0),
                dict(eps=math.inf)):
        assert go(residual(**bad)) == B.ERR_ARG, bad
    assert go(residual(d=8193)) == B.ERR_TOO_LARGE and go(residual(rows=1 << 40)) == B.ERR_TOO_LARGE
    assert go(residual(pre_weight=FAKE + 2)) == B.ERR_ALIGN and go(residual(pre_rstd=FAKE + 1)) == B.ERR_ALIGN
    keep = [rows(stride=63), rows(p=FAKE + 1), rows(p=0)]
    assert go(residual(), x=keep[0]) == B.ERR_ARG and go(residual(), y=keep[1]) == B.ERR_ALIGN and go(residual(), u=keep[2]) == B.ERR_ARG
    assert go(residual(rows=0), x=0, y=0, z=0, u=0) == B.OK


def test_residual_backward():
    r = rows()
    sums = lambda **kw: (ctypes.c_int64 * 5)(*(kw.get(k, 0) for k in ("w1", "b1", "gate", "w2", "b2")))  # noqa: E731
    go = lambda s, k=None, ws=FAKE, n=1 << 30, du=r: B.lib().a2sgd_residual_norm_backward(  # noqa: E731
        at(s), at(r), at(du), at(r), at(r), at(r), at(r), at(k) if k is not None else None, ws, n, 0, None)
    assert go(residual()) == B.ERR_ARG                                                      # no pre_rstd
    assert go(residual(pre_rstd=FAKE, flags=0)) == B.ERR_ARG                                # no pre_mean
    assert go(residual(pre_rstd=FAKE, flags=B.RESIDUAL_RMS | B.RESIDUAL_POST_NORM)) == B.ERR_ARG   # no post_rstd
    good = residual(pre_rstd=FAKE)
    for bad in (sums(w1=FAKE), sums(b1=FAKE), sums(gate=FAKE)):
        assert go(good, bad) == B.ERR_ARG
    assert go(good, sums(w2=FAKE), ws=None, n=0) == B.ERR_ARG and go(good, sums(w2=FAKE), n=64) == B.ERR_ARG
    assert go(good, sums(w2=FAKE + 1)) == B.ERR_ALIGN and go(good, sums(w2=FAKE), ws=FAKE + 16) == B.ERR_ALIGN
