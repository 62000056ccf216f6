"""Rotary positions with several axes against their definition in 64 bits, through the binding."""
import math
from fractions import Fraction

import pytest
import torch

from paper_2006_07405_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def rows(gen, tokens, heads, d, dtype, pad=0, skew=0):
    buf = torch.full((tokens * (heads * d + pad) + skew,), math.nan, dtype=dtype, device="cuda")
    view = buf.as_strided((tokens, heads, d), (heads * d + pad, d, 1), skew)
    view.copy_(torch.empty((tokens, heads, d), device="cuda").normal_(generator=gen))
    return buf, view


def reference(x, positions, sections, base, interleaved, ladders, inverse):
    n, y = sum(sections), x.double().clone()
    pairs = [(a, l / s if ladders else None) for a, s in enumerate(sections) for l in range(s)]
    for j, (a, power) in enumerate(pairs):
        angle = positions[a].double() * base ** -(j / n if power is None else power)
        c, s = angle.cos()[:, None], angle.sin()[:, None] * (-1 if inverse else 1)
        i0, i1 = (2 * j, 2 * j + 1) if interleaved else (j, j + n)
        u, v = x[..., i0].double(), x[..., i1].double()
        y[..., i0], y[..., i1] = u * c - v * s, u * s + v * c
    return y


def check(got, want, x, far, dtype):
    """The sine and cosine are off by at most 2^-23 (two units of fp32, and 2^-33 of a turn), the 64-bit reference's angle by
    far * 2^-52, both sums of two products by 2^-23 of |u| + |v|, and the result by half a step of its type."""
    size = x.double().abs().amax(-1, keepdim=True) * 2
    bound = HALF_STEP[dtype] * want.abs() + (2.0 ** -22 + far * 2.0 ** -52) * size + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    assert ((got.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens, hq, hk, d, sections, pad, skew", [
    (1, 1, 0, 2, [1], 0, 0), (7, 3, 1, 64, [32], 0, 0), (33, 4, 2, 128, [16, 24, 24], 0, 0), (300, 25, 25, 64, [10, 11, 11], 8, 8),
    (65, 2, 2, 80, [20, 16], 3, 0), (65, 2, 1, 96, [8, 8], 0, 0), (40, 5, 1, 50, [3, 4, 5, 6], 1, 1), (9, 2, 2, 512, [256], 0, 0),
    (1000, 1, 1, 17, [8], 0, 0)])
def test_against_the_definition(dtype, interleaved, tokens, hq, hk, d, sections, pad, skew):
    gen, dt = torch.Generator("cuda").manual_seed(tokens), DT[dtype]
    for ladders in (False, True):
        for inverse in (False, True):
            qb, q = rows(gen, tokens, hq, d, dt, pad, skew)
            k = rows(gen, tokens, hk, d, dt, pad, skew)[1] if hk else None
            pos = torch.randint(-5000, 100000, (len(sections), tokens), generator=gen, device="cuda", dtype=torch.int32)
            ob, qo = rows(gen, tokens, hq, d, dt, pad, skew)
            guard = torch.isnan(ob)
            ko = rows(gen, tokens, hk, d, dt, pad, skew)[1] if hk else None
            how = dict(base=10000.0, interleaved=interleaved, ladder_per_axis=ladders, inverse=inverse)
            B.a2sgd_rotary(q, k, qo, ko, pos, sections, **how)
            assert torch.equal(torch.isnan(ob), guard)
            for x, y in ((q, qo), (k, ko)):
                if x is not None:
                    check(y, reference(x, pos, sections, 10000.0, interleaved, ladders, inverse), x, 100000, dt)
                    n = 2 * sum(sections)
                    assert torch.equal(y[..., n:], x[..., n:])
            keep = q.clone()
            B.a2sgd_rotary(q, k, q, k, pos, sections, **how)       # in place: the same bits
            assert torch.equal(q, qo) and (k is None or torch.equal(k, ko))
            B.a2sgd_rotary(keep, None, keep, None, pos, sections, **how)
            assert torch.equal(keep, qo)


def test_inverse_undoes_it():
    gen = torch.Generator("cuda").manual_seed(0)
    _, q = rows(gen, 100, 4, 64, torch.float32)
    pos = torch.randint(0, 1 << 30, (3, 100), generator=gen, device="cuda", dtype=torch.int32)
    a, b = torch.empty_like(q), torch.empty_like(q)
    B.a2sgd_rotary(q, None, a, None, pos, [8, 12, 12])
    B.a2sgd_rotary(a, None, b, None, pos, [8, 12, 12], inverse=True)
    assert ((b - q).abs() <= 2.0 ** -21 * 2 * q.abs().amax(-1, keepdim=True)).all()


def test_far_positions_exactly():
    """Whole fractions of a turn at positions near 2^31: the frequency's 64 bits are what counts."""
    base = 3.7
    pos = torch.tensor([[2147483647, -2147483648, 2000000011, 1, 0]], dtype=torch.int32, device="cuda")
    q = torch.zeros((5, 1, 6), device="cuda")
    q[..., :3] = 1.0            # (u, v) = (1, 0): the outputs are the cosine and the sine
    out = torch.empty_like(q)
    B.a2sgd_rotary(q, None, out, None, pos, [3], base=base)
    # 2 pi to 200 bits
    turn = Fraction(2 * 314159265358979323846264338327950288419716939937510582097494459230781640628620899, 10 ** 80)
    for t, p in enumerate(pos[0].tolist()):
        omega = Fraction(1)
        for j in range(3):
            part = (p * omega / turn) % 1
            angle = float(part) * 2.0 * math.pi
            # the frequency is held to 2^-63 of itself: position * omega * 2^-62 radians
            slack = 2.0 ** -22 + abs(p) * 2.0 ** -58
            assert abs(out[t, 0, j].item() - math.cos(angle)) <= slack and abs(out[t, 0, j + 3].item() - math.sin(angle)) <= slack
            # base^(-(j + 1) / 3) to 80 digits by Newton's iteration
            x = Fraction(base) ** (j + 1)
            r = Fraction(float(x) ** (1.0 / 3.0))
            for _ in range(3):
                r = (r - (r ** 3 - x) / (3 * r ** 2)).limit_denominator(10 ** 60)
            omega = 1 / r


def test_gradient_is_the_inverse():
    """<dy, rotate(x)> = <inverse(dy), x>, by differences that are exact because the map is linear."""
    gen = torch.Generator("cuda").manual_seed(3)
    (_, x), (_, dy) = rows(gen, 50, 3, 64, torch.float32), rows(gen, 50, 3, 64, torch.float32)
    pos = torch.randint(0, 5000, (2, 50), generator=gen, device="cuda", dtype=torch.int32)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    B.a2sgd_rotary(x, None, y, None, pos, [20, 12], ladder_per_axis=True)
    B.a2sgd_rotary(dy, None, dx, None, pos, [20, 12], ladder_per_axis=True, inverse=True)
    a, b = (dy.double() * y.double()).sum().item(), (dx.double() * x.double()).sum().item()
    # every element carries 2^-21 of its pair's size at most, on either side
    assert abs(a - b) <= 4 * 2.0 ** -21 * (dy.double().abs().amax(-1) * x.double().abs().amax(-1)).sum().item() * 64


def test_captured():
    gen = torch.Generator("cuda").manual_seed(3)
    (_, x), (_, other) = rows(gen, 50, 3, 64, torch.bfloat16), rows(gen, 50, 3, 64, torch.bfloat16)
    pos = torch.arange(50, device="cuda", dtype=torch.int32)[None].contiguous()
    want, y = torch.empty_like(x), torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.a2sgd_rotary(x, None, y, None, pos, [32])
    x.copy_(other)
    graph.replay()
    B.a2sgd_rotary(other, None, want, None, pos, [32])
    assert torch.equal(want, y)


def test_refusals():
    q = torch.zeros((4, 2, 64), device="cuda")
    pos = torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    go = lambda **kw: B.a2sgd_rotary(**{**dict(q=q, k=q, q_out=q, k_out=q, positions=pos, sections=[16, 16]), **kw})  # noqa: E731
    go()
    for bad in (dict(q=q[0]), dict(k=None), dict(k_out=None), dict(positions=pos[:1]), dict(positions=pos.long()), dict(sections=[16, 0]),
                dict(sections=[]), dict(q_out=q.half()), dict(k=q[:2], k_out=q[:2]), dict(q=q.cpu()), dict(q=q.transpose(1, 2), q_out=q.transpose(1, 2)),
                dict(k=torch.zeros((4, 2, 32), device="cuda"), k_out=torch.zeros((4, 2, 32), device="cuda"))):
        with pytest.raises(ValueError):
            go(**bad)
    for bad in (dict(sections=[16, 17]), dict(base=0.0), dict(base=math.inf), dict(q_out=q[:, :1].expand(-1, 2, -1))):
        with pytest.raises(B.A2SGDError) as e:
            go(**bad)
        assert e.value.status == B.ERR_ARG
    with pytest.raises(B.A2SGDError) as e:
        wide = torch.zeros((4, 1, 514), device="cuda")
        go(q=wide, q_out=wide, k=None, k_out=None)
    assert e.value.status == B.ERR_TOO_LARGE
    five = torch.zeros((5, 4), dtype=torch.int32, device="cuda")
    with pytest.raises(B.A2SGDError) as e:
        go(positions=five, sections=[1, 1, 1, 1, 1])
    assert e.value.status == B.ERR_ARG
    empty = torch.empty((0, 2, 64), device="cuda")
    B.a2sgd_rotary(empty, None, empty, None, torch.empty((1, 0), dtype=torch.int32, device="cuda"), [32])
