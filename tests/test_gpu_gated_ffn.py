"""The gated feed-forward block through the binding, against the formulas in 64 bits and differences.

Tolerances.  Products of 16-bit numbers are exact in fp32.  A sum over k is accumulated 16 terms at a time in
fp32 registers that may truncate: each of the k / 16 steps, and the addition of its 16 terms, is off by at most
2^-22 of the absolute sum so far, so acc(k) = (k / 16 + 2) 2^-22 sum |terms|.  A rounding to the type is half a unit in
the last place, h_ulp.  act and act' by fast exponential and division: within (4 + 2 |a|) 2^-22 of |a| + 1.
 forward   a, b: acc(d), rounded.  hidden: the errors of a and b before their rounding, times the other factor (|act'| <= 1.2),
           that of act, rounded.  y, from the hidden that was written: acc(f), rounded.
 backward  dh: acc(d).  da, db: its error times |b act'|, |act|, act's error, rounded once (they are read back in the
           16-bit type).  dx, dw: those errors through the sums' absolute values, acc(k), rounded."""
import numpy as np
import pytest
import torch

from paper_2006_07405_b200 import binding as B

pytestmark = pytest.mark.gpu
HALF_ULP = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float16)}
TINY = {torch.bfloat16: 1e-37, torch.float16: 2.0 ** -25}     # below the normal range the unit is absolute


def _acc(k):
    return (k / 16 + 2) * 2.0 ** -22


def _act64(a, name):
    if name == "silu":
        p = torch.sigmoid(a)
        return a * p, p * (1 + a * (1 - p))
    k = np.sqrt(2 / np.pi)
    t = torch.tanh(k * (a + 0.044715 * a ** 3))
    return 0.5 * a * (1 + t), 0.5 * (1 + t) + 0.5 * a * (1 - t * t) * k * (1 + 3 * 0.044715 * a * a)


def _e_act(a):
    return (4 + 2 * a.abs()) * 2.0 ** -22 * (a.abs() + 1)


class Block:
    def __init__(self, t, d, f, dtype, pad=0, skew=0, seed=0, scale=1.0):
        gen = torch.Generator("cuda").manual_seed(seed)
        self.t, self.d, self.f, self.dtype, self.pad, self.skew = t, d, f, dtype, pad, skew
        self.bufs = {}
        rnd = lambda r, c, s: torch.empty((r, c), device="cuda").normal_(0, s, generator=gen)  # noqa: E731
        self.x = self.rows("x", rnd(t, d, scale))
        self.dy = self.rows("dy", rnd(t, d, 1.0))
        self.wg, self.wu = self.rows("wg", rnd(f, d, d ** -0.5)), self.rows("wu", rnd(f, d, d ** -0.5))
        self.wd = self.rows("wd", rnd(d, f, f ** -0.5))

    def rows(self, name, values):
        r, c = values.shape
        buf = torch.full((r * (c + self.pad) + self.skew,), 9.0, device="cuda").to(self.dtype)
        out = buf[self.skew:].view(r, c + self.pad)[:, :c]
        out.copy_(values)
        self.bufs[name] = buf
        return out

    def out(self, name, r, c):
        return self.rows(name, torch.full((r, c), float("nan"), device="cuda"))

    def check_edges(self):
        """Nothing outside the matrices was written."""
        for name, buf in self.bufs.items():
            c = self.f if name in ("a", "b", "h", "wd", "dwd") else self.d
            assert torch.all(buf[:self.skew] == 9.0)
            if self.pad and buf.numel() > self.skew:
                assert torch.all(buf[self.skew:].view(-1, c + self.pad)[:, c:] == 9.0), name

    def forward(self, act, train=True, stream=None):
        t, d, f = self.t, self.d, self.f
        self.y, self.h = self.out("y", t, d), self.out("h", t, f)
        self.a, self.b = (self.out("a", t, f), self.out("b", t, f)) if train else (None, None)
        work = torch.empty(B.a2sgd_gated_ffn_workspace(t, d, f), dtype=torch.uint8, device="cuda")
        torch.cuda.current_stream().synchronize()
        B.a2sgd_gated_ffn_forward(self.x, self.wg, self.wu, self.wd, self.y, self.h, self.a, self.b, activation=act,
                                  workspace=work, stream=stream)
        assert B.a2sgd_gated_ffn_status(stream=stream) == B.OK

    def backward(self, act, only=("dx", "dwg", "dwu", "dwd"), stream=None):
        t, d, f = self.t, self.d, self.f
        shapes = {"dx": (t, d), "dwg": (f, d), "dwu": (f, d), "dwd": (d, f)}
        got = {k: self.out(k, *shapes[k]) if k in only else None for k in shapes}
        work = torch.empty(B.a2sgd_gated_ffn_workspace(t, d, f, backward=True), dtype=torch.uint8, device="cuda")
        torch.cuda.current_stream().synchronize()
        B.a2sgd_gated_ffn_backward(self.dy, self.x, self.wg, self.wu, self.wd, self.h, self.a, self.b, got["dx"], got["dwg"],
                                   got["dwu"], got["dwd"], activation=act, workspace=work, stream=stream)
        assert B.a2sgd_gated_ffn_status(stream=stream) == B.OK
        return got


def _within(got, ref, tol, what):
    u = HALF_ULP[got.dtype]
    tol = (tol + u * ref.abs()) * (1 + u) + TINY[got.dtype]
    err = (got.double() - ref).abs()
    assert torch.all(err <= tol), f"{what}: {(err / tol).max().item():.3g} times the tolerance, {int((~(err <= tol)).sum())} of {err.numel()}"


def _check_forward(p, act):
    x, wg, wu, wd = (t.double() for t in (p.x, p.wg, p.wu, p.wd))
    a, b = x @ wg.T, x @ wu.T
    ea, eb = _acc(p.d) * (x.abs() @ wg.abs().T), _acc(p.d) * (x.abs() @ wu.abs().T)
    if p.a is not None:
        _within(p.a, a, ea, "a")
        _within(p.b, b, eb, "b")
    value, _ = _act64(a, act)
    eh = (1.2 * ea + _e_act(a)) * (b.abs() + eb) + value.abs() * eb
    _within(p.h, value * b, eh, "hidden")
    h = p.h.double()
    _within(p.y, h @ wd.T, _acc(p.f) * (h.abs() @ wd.abs().T), "y")


def _check_backward(p, act, got):
    x, wg, wu, wd, dy, h, a, b = (t.double() for t in (p.x, p.wg, p.wu, p.wd, p.dy, p.h, p.a, p.b))
    u = HALF_ULP[p.dtype]
    dh = dy @ wd
    e = _acc(p.d) * (dy.abs() @ wd.abs())
    value, slope = _act64(a, act)
    da, db = dh * b * slope, dh * value
    eda = (e * (slope.abs() + _e_act(a)) + dh.abs() * _e_act(a)) * b.abs() + 2.0 ** -22 * da.abs()
    edb = e * (value.abs() + _e_act(a)) + dh.abs() * _e_act(a) + 2.0 ** -22 * db.abs()
    eda, edb = eda + u * (da.abs() + eda) + TINY[p.dtype], edb + u * (db.abs() + edb) + TINY[p.dtype]
    if got["dx"] is not None:
        tol = eda @ wg.abs() + edb @ wu.abs() + _acc(2 * p.f) * (da.abs() @ wg.abs() + db.abs() @ wu.abs())
        _within(got["dx"], da @ wg + db @ wu, tol, "dx")
    for name, left, err, right in (("dwg", da, eda, x), ("dwu", db, edb, x), ("dwd", dy, torch.zeros_like(dy), h)):
        if got[name] is not None:
            _within(got[name], left.T @ right, err.T @ right.abs() + _acc(p.t) * (left.abs().T @ right.abs()), name)


SHAPES = [(1, 64, 64), (1, 1600, 6400), (3, 8, 16), (5, 1, 1), (17, 72, 200), (128, 128, 128), (129, 130, 131), (256, 256, 256),
          (300, 200, 520), (257, 777, 300), (1000, 64, 1000), (31, 520, 1030), (2, 1003, 2050), (600, 1600, 640), (2100, 512, 1408)]


@pytest.mark.parametrize("t,d,f", SHAPES)
@pytest.mark.parametrize("dtype,act", [(torch.bfloat16, "silu"), (torch.float16, "gelu_tanh")])
@pytest.mark.parametrize("pad,skew", [(0, 0), (8, 8), (3, 1)])
def test_forward_and_backward(t, d, f, dtype, act, pad, skew):
    p = Block(t, d, f, dtype, pad, skew)
    p.forward(act)
    _check_forward(p, act)
    _check_backward(p, act, p.backward(act))
    p.check_edges()


@pytest.mark.parametrize("t,d,f,pad", [(70, 777, 1001, 7), (300, 1601, 321, 7), (1, 9, 17, 7), (5, 1, 1, 7), (260, 130, 66, 6), (3, 61, 2045, 3)])
def test_rows_of_odd_length_at_aligned_addresses(t, d, f, pad):
    p = Block(t, d, f, torch.bfloat16, pad, 8)
    p.forward("silu")
    _check_forward(p, "silu")
    _check_backward(p, "silu", p.backward("silu"))
    p.check_edges()


@pytest.mark.parametrize("t,d,f", [(1300, 1600, 640), (2500, 1344, 256), (9600, 512, 128), (4736, 1024, 192), (3000, 2048, 64),
                                   (40, 1600, 4096), (700, 200, 8192)])
def test_every_tile_width_and_split(t, d, f):
    """Sizes whose best tiles are 64 to 512 columns wide, whole and split in depth."""
    p = Block(t, d, f, torch.bfloat16)
    p.forward("silu")
    _check_forward(p, "silu")
    _check_backward(p, "silu", p.backward("silu"))


@pytest.mark.parametrize("dtype,act", [(torch.bfloat16, "gelu_tanh"), (torch.float16, "silu")])
@pytest.mark.parametrize("t", [1, 2, 7, 8, 9, 16, 17, 33, 64, 65])
def test_few_tokens_without_what_the_backward_pass_needs(t, dtype, act):
    for pad in (0, 1):
        p = Block(t, 328, 1100, dtype, pad, seed=t)
        p.forward(act, train=False)
        _check_forward(p, act)
        p.check_edges()


@pytest.mark.parametrize("only", [("dx",), ("dwg",), ("dwu", "dwd"), ("dwd",), ()])
def test_parts_of_the_backward_pass(only):
    p = Block(200, 136, 264, torch.bfloat16)
    p.forward("silu")
    got, part = p.backward("silu"), p.backward("silu", only)
    for k in got:
        assert (part[k] is None) == (k not in only)
        if part[k] is not None:
            assert torch.equal(part[k], got[k])


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_large_preactivations(act):
    """Up to where the type ends: the activation saturates to a or 0 and nothing turns to NaN."""
    p = Block(64, 64, 128, torch.bfloat16, scale=100.0)
    p.forward(act)
    _check_forward(p, act)
    got = p.backward(act)
    assert all(torch.isfinite(g).all() for g in got.values())
    p.a.fill_(-3e30)
    p.a[:, ::2] = 3e30
    got = p.backward(act, only=("dwu",))                      # db = dh act(a): finite or overflowed, never NaN from 0 * inf
    p.dy.fill_(1e-30)
    got = p.backward(act)
    assert all(torch.isfinite(g).all() for g in got.values())


def test_a_token_that_is_not_finite_stays_in_its_row():
    p, q = Block(300, 136, 264, torch.bfloat16), Block(300, 136, 264, torch.bfloat16)
    p.x[140, 3] = float("nan")
    p.forward("silu")
    q.forward("silu")
    keep = torch.arange(300, device="cuda") != 140
    assert torch.isnan(p.y[140]).all() and torch.equal(p.y[keep], q.y[keep]) and torch.equal(p.h[keep], q.h[keep])


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_gradients_against_differences(act):
    """f = sum(dy y) along random directions, by central differences in 64 bits (their own error: h^2 = 1e-8 of a third
    derivative of order one).  The kernels' errors are roundings to 11 bits, independent of one another: of da and db, of
    the inputs hidden, gate and up, and of the result, together under 4 * 2^-11 of each term; along a random direction
    they add up like the terms themselves, in the root mean square: 4 * 2^-11 * sqrt(sum (g v)^2) has a factor of 8 to
    spare for the tail."""
    p = Block(40, 72, 104, torch.float16, seed=5)
    p.forward(act)
    got = p.backward(act)
    x, wg, wu, wd, dy = (t.double() for t in (p.x, p.wg, p.wu, p.wd, p.dy))

    def f(x, wg, wu, wd):
        return (dy * ((_act64(x @ wg.T, act)[0] * (x @ wu.T)) @ wd.T)).sum().item()

    gen = torch.Generator("cuda").manual_seed(1)
    for i, name in enumerate(("dx", "dwg", "dwu", "dwd")):
        for _ in range(4):
            args = [x, wg, wu, wd]
            v = torch.empty_like(args[i]).normal_(generator=gen)
            h = 1e-4
            up, down = list(args), list(args)
            up[i], down[i] = args[i] + h * v, args[i] - h * v
            g = got[name].double() * v
            tol = 8 * 4 * 2.0 ** -11 * g.square().sum().sqrt().item() + 1e-5 * g.abs().sum().item()
            assert abs((f(*up) - f(*down)) / (2 * h) - g.sum().item()) <= tol


def test_same_bits_every_time_and_on_another_stream():
    p = Block(1000, 520, 1030, torch.bfloat16, 3, 1)
    outs = []
    for stream in (None, None, torch.cuda.Stream()):
        p.forward("silu", stream=stream)
        got = p.backward("silu", stream=stream)
        outs.append([t.clone() for t in (p.y, p.h, p.a, p.b, *got.values())])
    for other in outs[1:]:
        for a, b in zip(outs[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("t", [12, 40, 300])
def test_less_workspace_means_no_splitting(t):
    """Aligned matrices need no workspace forward, and only da and db backward; what is then not split is as right."""
    p = Block(t, 1600, 2048, torch.bfloat16)
    p.y, p.h, p.a, p.b = p.out("y", t, 1600), p.out("h", t, 2048), p.out("a", t, 2048), p.out("b", t, 2048)
    B.a2sgd_gated_ffn_forward(p.x, p.wg, p.wu, p.wd, p.y, p.h, p.a, p.b)
    _check_forward(p, "silu")
    got = {"dx": p.out("dx", t, 1600), "dwg": p.out("dwg", 2048, 1600), "dwu": p.out("dwu", 2048, 1600), "dwd": p.out("dwd", 1600, 2048)}
    room = -(-t * 2048 * 2 // 256) * 256
    work = torch.empty(2 * room, dtype=torch.uint8, device="cuda")
    B.a2sgd_gated_ffn_backward(p.dy, p.x, p.wg, p.wu, p.wd, p.h, p.a, p.b, *got.values(), workspace=work)
    assert B.a2sgd_gated_ffn_status() == B.OK
    _check_backward(p, "silu", got)


def test_calls_can_be_captured_in_a_graph():
    """A captured forward and backward pass replays to the same bits."""
    p = Block(200, 264, 520, torch.bfloat16)
    p.forward("silu")
    got = p.backward("silu")
    want = [t.clone() for t in (p.y, p.h, *got.values())]
    y, h, a, b = p.out("y", 200, 264), p.out("h", 200, 520), p.out("a", 200, 520), p.out("b", 200, 520)
    grads = [torch.zeros_like(g) for g in got.values()]
    work = torch.empty(B.a2sgd_gated_ffn_workspace(200, 264, 520, backward=True), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.a2sgd_gated_ffn_forward(p.x, p.wg, p.wu, p.wd, y, h, a, b, workspace=work)
        B.a2sgd_gated_ffn_backward(p.dy, p.x, p.wg, p.wu, p.wd, h, a, b, *grads, workspace=work)
    for _ in range(2):
        for t in (y, h, a, b, *grads):
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        for x, ref in zip((y, h, *grads), want):
            assert torch.equal(x, ref)


def test_no_tokens_and_refusals():
    p = Block(0, 64, 128, torch.bfloat16)
    p.forward("silu")
    got = p.backward("silu")
    assert all(torch.all(got[k] == 0) for k in ("dwg", "dwu", "dwd"))
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    t, d, f = 4, 64, 128
    good = dict(x=z(t, d), w_gate=z(f, d), w_up=z(f, d), w_down=z(d, f), y=z(t, d), hidden=z(t, f), gate=z(t, f), up=z(t, f))
    B.a2sgd_gated_ffn_forward(**good)
    for bad in (dict(x=z(t, d).cpu()), dict(x=z(t, d, dtype=torch.float32)), dict(w_up=z(f + 1, d)), dict(w_down=z(f, d)),
                dict(y=z(t, d, dtype=torch.float16)), dict(gate=None), dict(up=None), dict(activation="relu"),
                dict(w_gate=z(f, 2 * d)[:, ::2]), dict(x=z(1, d).expand(t, d)), dict(y=z(t + 1, d)), dict(hidden=z(t, f)[0])):
        with pytest.raises((ValueError, B.A2SGDError)):
            B.a2sgd_gated_ffn_forward(**{**good, **bad})
    odd = z(t, d + 1)[:, :d]                                   # needs its copy, and there is no workspace
    with pytest.raises(B.A2SGDError) as e:
        B.a2sgd_gated_ffn_forward(**{**good, "x": odd})
    assert e.value.status == B.ERR_ARG
    with pytest.raises(B.A2SGDError) as e:                     # da and db need room
        B.a2sgd_gated_ffn_backward(good["y"], good["x"], good["w_gate"], good["w_up"], good["w_down"], good["hidden"], good["gate"],
                                   good["up"], z(t, d), None, None, None)
    assert e.value.status == B.ERR_ARG
    n = B.a2sgd_gated_ffn_workspace(t, d, f, backward=True, aligned=True)
    work = torch.empty(n, dtype=torch.uint8, device="cuda")
    B.a2sgd_gated_ffn_backward(good["y"], good["x"], good["w_gate"], good["w_up"], good["w_down"], good["hidden"], good["gate"],
                               good["up"], z(t, d), z(f, d), z(f, d), z(d, f), workspace=work)
    torch.cuda.synchronize()
