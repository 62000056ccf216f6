"""Cases that measure the operators of the attention half of a block: attention with a sliding window and first tokens that
stay visible (forward, backward, and few queries over a cache), rotary positions with several axes, and the residual
connection with its gate, its scale and the norms before and after it.

``run`` computes them in plain torch operations, or, where ``own`` is set, with this package's kernels.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
NORM_EPS = 1e-5


# ----------------------------------------------------------------- the cases
def listed():
    return [
        # the next token of four texts, a small model's heads: latency
        {"name": "attn_decode_4x25x64", "op": "attn_fwd", "layout": "cache", "seqs": 4, "q": 1, "k": 2048, "hq": 25, "hkv": 25,
         "d": 64, "window": 1024, "sinks": 4, "dtype": "bf16", "pad": 0, "train": False},
        # the next token of a full serving batch with shared key heads: the cache's bytes count
        {"name": "attn_decode_64x32x128", "op": "attn_fwd", "layout": "cache", "seqs": 64, "q": 1, "k": 8192, "hq": 32, "hkv": 8,
         "d": 128, "window": 4096, "sinks": 16, "dtype": "bf16", "pad": 0, "train": False},
        # a training batch of the benchmark's 25 heads of 64, forward with what the backward pass needs
        {"name": "attn_fwd_8x4096x25x64", "op": "attn_fwd", "layout": "dense", "seqs": 8, "q": 4096, "k": 4096, "hq": 25, "hkv": 25,
         "d": 64, "window": 1024, "sinks": 4, "dtype": "bf16", "pad": 0, "train": True},
        # documents of all lengths packed one behind another, shared key heads, a window longer than most of them
        {"name": "attn_fwd_packed_20011x16x128", "op": "attn_fwd", "layout": "packed", "seqs": 13, "q": 20011, "k": 20011, "hq": 16,
         "hkv": 4, "d": 128, "window": 4096, "sinks": 0, "dtype": "f16", "pad": 0, "train": True},
        {"name": "attn_bwd_8x4096x25x64", "op": "attn_bwd", "layout": "dense", "seqs": 8, "q": 4096, "k": 4096, "hq": 25, "hkv": 25,
         "d": 64, "window": 1024, "sinks": 4, "dtype": "bf16", "pad": 0},
        # packed odd lengths, a head length between the tiles', more first tokens than a tile has
        {"name": "attn_bwd_packed_5003x12x80", "op": "attn_bwd", "layout": "packed", "seqs": 7, "q": 5003, "k": 5003, "hq": 12,
         "hkv": 4, "d": 80, "window": 300, "sinks": 130, "dtype": "f16", "pad": 0},
        # a handful of tokens of text: latency
        {"name": "rotary_16x25x64", "op": "rotary", "tokens": 16, "hq": 25, "hkv": 25, "d": 64, "sections": "32", "interleaved": True,
         "ladders": False, "inverse": False, "dtype": "bf16", "pad": 0},
        # frames of video: time, height and width, no multiple of eight of them
        {"name": "rotary_65531x32x128_video", "op": "rotary", "tokens": 65531, "hq": 32, "hkv": 8, "d": 128, "sections": "16,24,24",
         "interleaved": False, "ladders": False, "inverse": False, "dtype": "bf16", "pad": 0},
        # an image's rows and columns, a ladder of frequencies for each, part of the head turned, backward, odd rows
        {"name": "rotary_4097x13x80_image", "op": "rotary", "tokens": 4097, "hq": 13, "hkv": 13, "d": 80, "sections": "20,16",
         "interleaved": False, "ladders": True, "inverse": True, "dtype": "f32", "pad": 3},
        # a handful of tokens: latency
        {"name": "resnorm_fwd_16x1600", "op": "resnorm_fwd", "rows": 16, "d": 1600, "kind": "rms", "post": True, "gate_rows": 0,
         "dtype": "bf16", "residual": "bf16", "param": "f32", "pad": 0},
        # 64 samples of 1024 rows, a gate for each, the residual stream in fp32
        {"name": "resnorm_fwd_65536x1600", "op": "resnorm_fwd", "rows": 65536, "d": 1600, "kind": "rms", "post": True,
         "gate_rows": 1024, "dtype": "bf16", "residual": "f32", "param": "f32", "pad": 0},
        {"name": "resnorm_bwd_65536x1600", "op": "resnorm_bwd", "rows": 65536, "d": 1600, "kind": "layer", "post": True,
         "gate_rows": 65536, "dtype": "bf16", "residual": "bf16", "param": "bf16", "pad": 0},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _head_dim(rng):
    return rng.choice([64, 64, 64, 128, 128, 80, 96, 32, rng.randrange(8, 129)])


def _heads(rng):
    hkv = rng.choice([1, 2, 4, 8, 12, 25])
    return hkv * (1 if hkv > 8 else rng.choice([1, 1, 2, 3, 4])), hkv


def _draw_attention(rng):
    op = rng.choice(["decode", "attn_fwd", "attn_fwd", "attn_bwd", "attn_bwd"])
    hq, hkv = _heads(rng)
    d, pad = _head_dim(rng), rng.choice([0, 0, 0, 8, 3])
    case = {"op": op, "hq": hq, "hkv": hkv, "d": d, "sinks": rng.choice([0, 1, 4, 4, 16, 64, rng.randrange(0, 300)]),
            "dtype": rng.choice(["bf16", "bf16", "f16"]), "pad": pad}
    if op == "decode":
        k = _log_int(rng, 64, 16384)
        seqs = _log_int(rng, 1, max(1, min(64, (1 << 29) // (k * hkv * d))))
        case.update(op="attn_fwd", layout="cache", seqs=seqs, q=rng.choice([1, 1, 1, 1, 2, 5]), k=k, train=False)
    else:
        packed = rng.random() < 0.5
        rows = _log_int(rng, 64, 32768)
        seqs = _log_int(rng, 1, max(1, min(32, rows // 32)))
        if not packed:
            rows = max(1, rows // seqs)
        case.update(layout="packed" if packed else "dense", seqs=seqs, q=rows, k=rows)
        if op == "attn_fwd":
            case["train"] = rng.random() < 0.6
    case["window"] = _log_int(rng, 16, max(17, case["k"]))
    while _pairs(case) * hq * (128 if d > 64 else 64) > 800_000_000 * 64:
        case["window"] = max(16, case["window"] // 2)
        case["sinks"] //= 2
    return case


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "rotary", "resnorm_fwd", "resnorm_bwd"])
    if op == "attention":
        return _draw_attention(rng)
    if op == "rotary":
        hq, hkv = _heads(rng)
        d = 2 * rng.randrange(8, 65) if rng.random() < 0.3 else rng.choice([64, 128, 80, 96, 32])
        half, axes = (d if rng.random() < 0.7 else max(8, d // 2)) // 2, rng.choice([1, 2, 3, 3, 4])
        cuts = sorted(rng.randrange(1, half) for _ in range(axes - 1))
        sections = [b - a for a, b in zip([0] + cuts, cuts + [half])]
        dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
        most = max(1, 65536 * 40 * 256 // ((hq + hkv) * d * SIZES[dtype]))
        return {"op": op, "tokens": _log_int(rng, 1, min(65536, most)), "hq": hq, "hkv": hkv, "d": d,
                "sections": ",".join(str(s) for s in sections if s > 0), "interleaved": rng.random() < 0.4,
                "ladders": rng.random() < 0.4, "inverse": rng.random() < 0.5, "dtype": dtype, "pad": rng.choice([0, 0, 8, 3])}
    d = _log_int(rng, 16, 8192)
    if rng.random() < 0.7:
        d = max(8, d // 8 * 8)
    rows = _log_int(rng, 1, min(65536, 65536 * 1600 // d))
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    return {"op": op, "rows": rows, "d": d, "kind": rng.choice(["rms", "layer"]), "post": rng.random() < 0.8,
            "gate_rows": rng.choice([0, rows, max(1, rows // 7)]), "dtype": dtype, "residual": rng.choice(["f32", dtype]),
            "param": rng.choice(["f32", dtype]), "pad": rng.choice([0, 0, 8, 3])}


# ----------------------------------------------------------------- sequences
def _lengths(case):
    """(first query row, queries, first key row, keys) of each sequence, within its own plane or the packed rows."""
    n = case["seqs"]
    if case["layout"] == "dense":
        return [(0, case["q"], 0, case["k"])] * n
    if case["layout"] == "cache":
        # caches filled to different lengths, from half of their rows up
        return [(0, case["q"], 0, max(1, int(case["k"] * (0.5 + 0.5 * ((i * 0.6180339887498949 + 0.5) % 1.0))))) for i in range(n)]
    weight = [4.0 ** (2.0 * ((i * 0.6180339887498949 + 0.3) % 1.0)) for i in range(n)]
    size = [max(1, int(case["q"] * x / sum(weight))) for x in weight]
    size[max(range(n), key=size.__getitem__)] += case["q"] - sum(size)
    out, at = [], 0
    for s in size:
        out.append((at, s, at, s))
        at += s
    return out


def _ramp(a, b):
    """a + (a + 1) + ... + b, terms below 0 left out."""
    a = max(a, 0)
    return (a + b) * (b - a + 1) // 2 if b >= a else 0


def _visible(lq, lk, window, sinks):
    """Visible pairs of a sequence: window keys up to a query's own place, and first tokens before the window."""
    p0, p1 = lk - lq, lk - 1
    pairs = _ramp(p0 + 1, p1 + 1) - _ramp(p0 + 1 - window, p1 + 1 - window)
    return pairs + _ramp(p0 + 1 - window, p1 + 1 - window) - _ramp(p0 + 1 - window - sinks, p1 + 1 - window - sinks)


def _pairs(case):
    return sum(_visible(lq, lk, case["window"], case["sinks"]) for _, lq, _, lk in _lengths(case))


# ----------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(DEV).manual_seed(int(seed) % (1 << 62))


def _normal(gen, *shape, std=1.0):
    return torch.empty(shape, device=DEV).normal_(0.0, std, generator=gen)


def _heads_view(gen, lead, heads, d, dtype, pad):
    """[..., heads, d] inside rows that are ``pad`` elements wider; random values, or zeros without a generator."""
    shape = (*lead, heads * d + pad)
    buf = torch.zeros(shape, dtype=dtype, device=DEV) if gen is None else torch.empty(shape, dtype=dtype, device=DEV)
    view = buf[..., :heads * d].unflatten(-1, (heads, d))
    if gen is not None:
        view.copy_(torch.empty((*lead, heads, d), dtype=dtype, device=DEV).normal_(generator=gen))
    return view


def _sequences(s, *names):
    """For each run of sequences of equal lengths: fp32 [n, rows, heads, d] of each named tensor, and where it lies."""
    case = s["case"]
    if case["layout"] == "dense":
        yield slice(0, case["seqs"]), None, None, [s[x].float() for x in names]
        return
    for i, (q0, lq, k0, lk) in enumerate(s["lengths"]):
        which = slice(i, i + 1)
        cut = []
        for x in names:
            first, count = (k0, lk) if x in ("k", "v") else (q0, lq)
            t = s[x][first:first + count][None] if case["layout"] == "packed" else s[x][which, first:first + count]
            cut.append(t.float())
        yield which, (q0, lq), (k0, lk), cut


def _prepare_attention(case, seed):
    gen, dtype, d, pad = _gen(seed), DTYPES[case["dtype"]], case["d"], case["pad"]
    hq, hkv, n = case["hq"], case["hkv"], case["seqs"]
    lq, lk = ((case["q"],), (case["k"],)) if case["layout"] == "packed" else ((n, case["q"]), (n, case["k"]))
    s = {"case": case, "lengths": _lengths(case), "scale": d ** -0.5}
    if case["layout"] == "cache":
        s["q"] = _heads_view(gen, lq, hq, d, dtype, pad)
        s["k"], s["v"] = (_heads_view(gen, lk, hkv, d, dtype, pad) for _ in range(2))
    else:   # one projection's output, as a block computes it
        qkv = _heads_view(gen, lq, hq + 2 * hkv, d, dtype, pad)
        s["q"], s["k"], s["v"] = qkv[..., :hq, :], qkv[..., hq:hq + hkv, :], qkv[..., hq + hkv:, :]
    ranges = torch.tensor(s["lengths"], dtype=torch.int32, device=DEV)
    if case["layout"] == "packed":
        s["q_ranges"], s["k_ranges"] = ranges[:, :2].contiguous(), ranges[:, 2:].contiguous()
    elif case["layout"] == "cache":
        s["q_ranges"], s["k_ranges"] = None, ranges[:, 2:].contiguous()
    else:
        s["q_ranges"], s["k_ranges"] = None, None
    lse_shape = (hq, case["q"]) if case["layout"] == "packed" else (n, hq, case["q"])
    s["o"] = _heads_view(None, lq, hq, d, dtype, pad)
    s["lse"] = torch.zeros(lse_shape, device=DEV)
    if case["op"] == "attn_bwd":
        s["do"] = _heads_view(gen, lq, hq, d, dtype, pad)
        _plain_attention(s)     # what the forward pass of this step left behind
        grads = _heads_view(None, lq, hq + 2 * hkv, d, dtype, pad)
        s["dq"], s["dk"], s["dv"] = grads[..., :hq, :], grads[..., hq:hq + hkv, :], grads[..., hq + hkv:, :]
    if own:
        from paper_2006_07405_b200 import binding as B
        s["B"] = B
        s["work"] = torch.empty(B.a2sgd_window_attention_workspace(s["q"], s["k"], case["window"], case["sinks"], n,
                                                                   backward=case["op"] == "attn_bwd"),
                                dtype=torch.uint8, device=DEV)
    return s


def _sections(case):
    return [int(x) for x in case["sections"].split(",")]


def _prepare_rotary(case, seed):
    gen, dtype, pad, t = _gen(seed), DTYPES[case["dtype"]], case["pad"], case["tokens"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    qk = _heads_view(gen, (t,), hq + hkv, d, dtype, pad)
    axes = len(_sections(case))
    # a text's places; an image's rows and columns; a video's frames, rows and columns, far into a long one
    if axes == 1:
        pos = [torch.arange(t, device=DEV) + int(torch.randint(0, 1 << 17, (), generator=gen, device=DEV))]
    else:
        side = max(1, math.isqrt(t) if axes == 2 else round(t ** (1.0 / 3.0)))
        i = torch.arange(t, device=DEV) + int(torch.randint(0, 1 << 15, (), generator=gen, device=DEV))
        pos = [i // side ** (axes - 1 - a) % (side if a else 1 << 30) for a in range(axes)]
    out = _heads_view(None, (t,), hq + hkv, d, dtype, pad)
    s = {"case": case, "q": qk[:, :hq], "k": qk[:, hq:], "q_out": out[:, :hq], "k_out": out[:, hq:],
         "positions": torch.stack(pos).to(torch.int32).contiguous()}
    if own:
        from paper_2006_07405_b200 import binding as B
        s["B"] = B
    return s


def _rows(values, dtype, pad):
    """The values as rows of a buffer that is ``pad`` elements wider."""
    r, c = values.shape
    buf = torch.zeros((r, c + pad), dtype=dtype, device=DEV)
    buf[:, :c].copy_(values)
    return buf[:, :c]


def _prepare_resnorm(case, seed):
    gen = _gen(seed)
    rows, d, pad = case["rows"], case["d"], case["pad"]
    dtype, residual, param = DTYPES[case["dtype"]], DTYPES[case["residual"]], DTYPES[case["param"]]
    empty = lambda t: torch.zeros((rows, d + pad), dtype=t, device=DEV)[:, :d]  # noqa: E731
    groups = 0 if case["gate_rows"] == 0 else -(-rows // case["gate_rows"])
    s = {"case": case, "alpha": 0.7, "y": _rows(_normal(gen, rows, d) * _normal(gen, rows, 1, std=0.5).exp_() + _normal(gen, 1, d, std=0.3), dtype, pad),
         "w1": (1.0 + _normal(gen, d, std=0.2)).to(param) if case["post"] else None,
         "b1": _normal(gen, d, std=0.2).to(param) if case["post"] and case["kind"] == "layer" else None,
         "w2": (1.0 + _normal(gen, d, std=0.2)).to(param),
         "b2": _normal(gen, d, std=0.2).to(param) if case["kind"] == "layer" else None,
         "gate": _normal(gen, groups, d, std=0.5).to(param) if groups else None}
    s["x"] = _rows(_normal(gen, rows, d) * 2.0 + _normal(gen, 1, d), residual, pad)
    stat = lambda: torch.empty(rows, device=DEV)  # noqa: E731
    layer = case["kind"] == "layer"
    s.update(mean1=stat() if layer and case["post"] else None, rstd1=stat() if case["post"] else None,
             mean2=stat() if layer else None, rstd2=stat())
    s.update(z=empty(residual), u=empty(dtype))
    if case["op"] == "resnorm_bwd":
        for k, v in _plain_resnorm_fwd(s).items():     # what the forward pass left behind
            s[k].copy_(v)
        s.update(dz=_rows(_normal(gen, rows, d, std=0.5), residual, pad), du=_rows(_normal(gen, rows, d), dtype, pad),
                 dx=empty(residual), dy=empty(dtype))
        for k in ("w1", "b1", "w2", "b2", "gate"):
            s["d" + k] = None if s[k] is None else torch.empty_like(s[k])
    if own:
        from paper_2006_07405_b200 import binding as B
        s["B"] = B
        if case["op"] == "resnorm_bwd":
            s["work"] = torch.empty(B.a2sgd_residual_norm_workspace(rows, d, case["gate_rows"]), dtype=torch.uint8, device=DEV)
    return s


def prepare(case, seed):
    if case["op"].startswith("attn"):
        return _prepare_attention(case, seed)
    return _prepare_rotary(case, seed) if case["op"] == "rotary" else _prepare_resnorm(case, seed)


# ----------------------------------------------------------------- the plain forms
def _blocks(lq, lk, window, sinks, rows=512):
    """Blocks of queries, the keys that any of them sees, and which of those each sees."""
    for a in range(0, lq, rows):
        b = min(lq, a + rows)
        lo, hi = max(0, a + lk - lq - window + 1), b + lk - lq
        if hi <= 0:
            yield a, b, None, None
            continue
        first = min(sinks, lo)
        keys = torch.cat([torch.arange(first, device=DEV), torch.arange(lo, hi, device=DEV)])
        at = torch.arange(a, b, device=DEV)[:, None] + (lk - lq)
        yield a, b, keys, (keys <= at) & ((keys > at - window) | (keys < sinks))


def _by_heads(t, hkv):
    """[n, rows, heads, d] as [n, key heads, heads of each, rows, d]."""
    n, rows, h, d = t.shape
    return t.view(n, rows, hkv, h // hkv, d).permute(0, 2, 3, 1, 4)


def _put(s, name, which, rows, value):
    """[n, rows, heads, d] into the named output, rounded once."""
    layout = s["case"]["layout"]
    if layout == "dense":
        s[name].copy_(value)
    elif layout == "packed":
        s[name][rows[0]:rows[0] + rows[1]].copy_(value[0])
    else:
        s[name][which, rows[0]:rows[0] + rows[1]].copy_(value)


def _put_lse(s, which, rows, value):
    layout = s["case"]["layout"]
    if layout == "packed":
        s["lse"][:, rows[0]:rows[0] + rows[1]].copy_(value[0])
    else:
        s["lse"][which].copy_(value)


def _plain_attention(s):
    case, hkv = s["case"], s["case"]["hkv"]
    for which, q_at, _, (q, k, v) in _sequences(s, "q", "k", "v"):
        n, lq, hq, d = q.shape
        lk = k.shape[1]
        q, k, v = _by_heads(q, hkv), _by_heads(k, hkv), _by_heads(v, hkv)
        o = torch.zeros((n, lq, hq, d), device=DEV)
        lse = torch.full((n, hq, lq), -math.inf, device=DEV)
        for a, b, keys, seen in _blocks(lq, lk, case["window"], case["sinks"]):
            if keys is None:
                continue
            x = (q[:, :, :, a:b] @ k[:, :, :, keys].transpose(-1, -2)) * s["scale"]
            x = x.masked_fill(~seen, -math.inf)
            top = x.amax(-1, keepdim=True)
            top = torch.where(top == -math.inf, torch.zeros_like(top), top)
            p = (x - top).exp()
            total = p.sum(-1, keepdim=True)
            out = (p @ v[:, :, :, keys]) / torch.where(total > 0, total, torch.ones_like(total))
            o[:, a:b] = out.permute(0, 3, 1, 2, 4).reshape(n, b - a, hq, d)
            lse[:, :, a:b] = (total.log() + top).reshape(n, hq, b - a)
        _put(s, "o", which, q_at, o)
        _put_lse(s, which, q_at, lse)
    return {"o": s["o"], "lse": s["lse"]} if case.get("train") else {"o": s["o"]}


def _plain_attention_bwd(s):
    case, hkv = s["case"], s["case"]["hkv"]
    for which, q_at, k_at, (q, k, v, o, do) in _sequences(s, "q", "k", "v", "o", "do"):
        n, lq, hq, d = q.shape
        lk = k.shape[1]
        lse = s["lse"][None, :, q_at[0]:q_at[0] + lq] if case["layout"] == "packed" else s["lse"][which]
        lse = lse.reshape(n, hkv, hq // hkv, lq, 1)
        q, k, v, o, do = (_by_heads(t, hkv) for t in (q, k, v, o, do))
        delta = (o * do).sum(-1, keepdim=True)
        dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        for a, b, keys, seen in _blocks(lq, lk, case["window"], case["sinks"]):
            if keys is None:
                continue
            kk, vv, qq, gg = k[:, :, :, keys], v[:, :, :, keys], q[:, :, :, a:b], do[:, :, :, a:b]
            x = (qq @ kk.transpose(-1, -2)) * s["scale"] - lse[:, :, :, a:b]
            p = torch.where(seen, x.exp(), torch.zeros_like(x))
            ds = p * (gg @ vv.transpose(-1, -2) - delta[:, :, :, a:b]) * s["scale"]
            dq[:, :, :, a:b] = ds @ kk
            dk[:, :, :, keys] += (ds.transpose(-1, -2) @ qq).sum(2, keepdim=True)
            dv[:, :, :, keys] += (p.transpose(-1, -2) @ gg).sum(2, keepdim=True)
        rows = lambda t: t.permute(0, 3, 1, 2, 4).reshape(n, t.shape[3], -1, d)  # noqa: E731
        _put(s, "dq", which, q_at, rows(dq))
        _put(s, "dk", which, k_at, rows(dk))
        _put(s, "dv", which, k_at, rows(dv))
    return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


def _frequencies(case):
    """Radians a step of each pair, in 64 bits, and the axis that turns it."""
    sections = _sections(case)
    freq, axis, total = [], [], sum(sections)
    for a, n in enumerate(sections):
        for j in range(n):
            freq.append(10000.0 ** -(j / n if case["ladders"] else len(freq) / total))
            axis.append(a)
    return torch.tensor(freq, dtype=torch.float64, device=DEV), torch.tensor(axis, device=DEV)


def _plain_rotary(s):
    case = s["case"]
    freq, axis = _frequencies(case)
    angle = s["positions"].double()[axis].T * freq
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if case["inverse"]:
        sin = -sin
    half = freq.numel()
    for a, b in (("q", "q_out"), ("k", "k_out")):
        x = s[a].float()
        if case["interleaved"]:
            u, v = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
            turned = torch.stack([u * cos - v * sin, u * sin + v * cos], -1).flatten(-2)
        else:
            u, v = x[..., :half], x[..., half:2 * half]
            turned = torch.cat([u * cos - v * sin, u * sin + v * cos], -1)
        s[b].copy_(torch.cat([turned, x[..., 2 * half:]], -1))
    return {"q": s["q_out"], "k": s["k_out"]}


def _norm(x, kind):
    """The normalised rows, the mean (or None) and the reciprocal deviation."""
    mean = x.mean(1, keepdim=True) if kind == "layer" else None
    c = x if mean is None else x - mean
    rstd = 1.0 / (c.square().mean(1, keepdim=True) + NORM_EPS).sqrt()
    return c * rstd, mean, rstd


def _gate_rows(s):
    """The gate of each row, or 1."""
    if s["gate"] is None:
        return 1.0
    rows = s["case"]["rows"]
    return s["gate"].float()[torch.arange(rows, device=DEV) // s["case"]["gate_rows"]]


def _plain_resnorm_fwd(s):
    case, n, out = s["case"], s["y"].float(), {}
    if case["post"]:
        n, mean, rstd = _norm(n, case["kind"])
        n = n * s["w1"].float()
        if s["b1"] is not None:
            n = n + s["b1"].float()
            out["mean1"] = mean.view(-1)
        out["rstd1"] = rstd.view(-1)
    z = s["x"].float() + n * _gate_rows(s) * s["alpha"]
    u, mean, rstd = _norm(z, case["kind"])
    u = u * s["w2"].float()
    if s["b2"] is not None:
        u = u + s["b2"].float()
        out["mean2"] = mean.view(-1)
    return {**out, "rstd2": rstd.view(-1), "z": z.to(s["x"].dtype), "u": u.to(s["y"].dtype)}


def _plain_resnorm_bwd(s):
    case, out = s["case"], {}
    layer, pt = case["kind"] == "layer", s["w2"].dtype
    du, t = s["du"].float(), s["dz"].float()
    hat = (s["z"].float() - s["mean2"][:, None] if layer else s["z"].float()) * s["rstd2"][:, None]
    g = du * s["w2"].float()
    inner = g - hat * (g * hat).mean(1, keepdim=True)
    t = t + (inner - g.mean(1, keepdim=True) if layer else inner) * s["rstd2"][:, None]
    out["dw2"] = (du * hat).sum(0).to(pt)
    if layer:
        out["db2"] = du.sum(0).to(pt)
    out["dx"] = t.to(s["x"].dtype)
    dn, y = t * _gate_rows(s) * s["alpha"], s["y"].float()
    n = y
    if case["post"]:
        hat = (y - s["mean1"][:, None] if layer else y) * s["rstd1"][:, None]
        n = hat * s["w1"].float()
        out["dw1"] = (dn * hat).sum(0).to(pt)
        if layer:
            n = n + s["b1"].float()
            out["db1"] = dn.sum(0).to(pt)
        g = dn * s["w1"].float()
        inner = g - hat * (g * hat).mean(1, keepdim=True)
        dy = (inner - g.mean(1, keepdim=True) if layer else inner) * s["rstd1"][:, None]
    else:
        dy = dn
    out["dy"] = dy.to(s["y"].dtype)
    if s["gate"] is not None:
        groups, d = s["gate"].shape
        each = torch.zeros((groups * case["gate_rows"], d), device=DEV)
        each[:case["rows"]] = t * n * s["alpha"]
        out["dgate"] = each.view(groups, -1, d).sum(1).to(pt)
    return out


# ----------------------------------------------------------------- the framework's calls
def _own_attention(s):
    case = s["case"]
    s["B"].a2sgd_window_attention_forward(s["q"], s["k"], s["v"], s["o"], s["lse"] if case["train"] else None,
                                          window=case["window"], sinks=case["sinks"], scale=s["scale"],
                                          q_ranges=s["q_ranges"], k_ranges=s["k_ranges"], workspace=s["work"])
    return {"o": s["o"], "lse": s["lse"]} if case["train"] else {"o": s["o"]}


def _own_attention_bwd(s):
    case = s["case"]
    s["B"].a2sgd_window_attention_backward(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["dq"], s["dk"], s["dv"],
                                           window=case["window"], sinks=case["sinks"], scale=s["scale"],
                                           q_ranges=s["q_ranges"], k_ranges=s["k_ranges"], workspace=s["work"])
    return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


def _own_rotary(s):
    case = s["case"]
    s["B"].a2sgd_rotary(s["q"], s["k"], s["q_out"], s["k_out"], s["positions"], _sections(case), base=10000.0,
                        interleaved=case["interleaved"], ladder_per_axis=case["ladders"], inverse=case["inverse"])
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_resnorm_fwd(s):
    case = s["case"]
    s["B"].a2sgd_residual_norm_forward(s["x"], s["y"], s["z"], s["u"], kind=case["kind"], post=case["post"],
                                       post_weight=s["w1"], post_bias=s["b1"], gate=s["gate"], gate_rows=case["gate_rows"],
                                       alpha=s["alpha"], pre_weight=s["w2"], pre_bias=s["b2"], post_mean=s["mean1"],
                                       post_rstd=s["rstd1"], pre_mean=s["mean2"], pre_rstd=s["rstd2"], eps=NORM_EPS)
    out = {"mean1": s["mean1"], "rstd1": s["rstd1"], "mean2": s["mean2"], "rstd2": s["rstd2"], "z": s["z"], "u": s["u"]}
    return {k: v for k, v in out.items() if v is not None}


def _own_resnorm_bwd(s):
    case = s["case"]
    s["B"].a2sgd_residual_norm_backward(s["dz"], s["du"], s["y"], s["z"], s["dx"], s["dy"], kind=case["kind"], post=case["post"],
                                        post_weight=s["w1"], post_bias=s["b1"], gate=s["gate"], gate_rows=case["gate_rows"],
                                        alpha=s["alpha"], pre_weight=s["w2"], post_mean=s["mean1"], post_rstd=s["rstd1"],
                                        pre_mean=s["mean2"], pre_rstd=s["rstd2"], dpost_weight=s["dw1"], dpost_bias=s["db1"],
                                        dgate=s["dgate"], dpre_weight=s["dw2"], dpre_bias=s["db2"], workspace=s["work"])
    out = {k: s[k] for k in ("dw2", "db2", "dx", "dw1", "db1", "dy", "dgate")}
    return {k: v for k, v in out.items() if v is not None}


def run(state):
    op = state["case"]["op"]
    if own:
        return {"attn_fwd": _own_attention, "attn_bwd": _own_attention_bwd, "rotary": _own_rotary,
                "resnorm_fwd": _own_resnorm_fwd, "resnorm_bwd": _own_resnorm_bwd}[op](state)
    return {"attn_fwd": _plain_attention, "attn_bwd": _plain_attention_bwd, "rotary": _plain_rotary,
            "resnorm_fwd": _plain_resnorm_fwd, "resnorm_bwd": _plain_resnorm_bwd}[op](state)


# ----------------------------------------------------------------- the work
def work(case):
    op, e = case["op"], SIZES[case["dtype"]]
    if op.startswith("attn"):
        hq, hkv, d = case["hq"], case["hkv"], case["d"]
        rows_q, rows_k = 0, 0
        for _, lq, _, lk in _lengths(case):
            first = lk - lq - case["window"] + 1      # the keys that some query sees: the first ones, and from here on
            rows_q += lq
            rows_k += lk - max(0, first) + min(case["sinks"], max(0, first))
        q, k = rows_q * hq * d * e, rows_k * hkv * d * e
        if op == "attn_fwd":
            return {"bytes": 2 * q + 2 * k + (4 * rows_q * hq if case["train"] else 0), "flops": 4 * d * hq * _pairs(case)}
        return {"bytes": 4 * q + 4 * k + 4 * rows_q * hq, "flops": 10 * d * hq * _pairs(case)}
    if op == "rotary":
        t, n = case["tokens"], case["tokens"] * (case["hq"] + case["hkv"]) * case["d"]
        return {"bytes": 2 * n * e + 4 * t * len(_sections(case)), "flops": 3 * n}
    rows, d, r, p = case["rows"], case["d"], SIZES[case["residual"]], SIZES[case["param"]]
    layer, post = case["kind"] == "layer", case["post"]
    vectors = (2 if layer else 1) * (2 if post else 1) + (0 if case["gate_rows"] == 0 else -(-rows // case["gate_rows"]))
    stats = 4 * rows * (2 if layer else 1) * (2 if post else 1)
    if op == "resnorm_fwd":
        return {"bytes": 2 * rows * d * (e + r) + vectors * d * p + stats, "flops": 14 * rows * d}
    return {"bytes": 3 * rows * d * (e + r) + 2 * vectors * d * p + stats, "flops": 28 * rows * d}


# ----------------------------------------------------------------- the definition in 64 bits
def _exact_attention(s):
    case, hq, hkv = s["case"], s["case"]["hq"], s["case"]["hkv"]
    backward = case["op"] == "attn_bwd"
    packed = case["layout"] == "packed"
    names = ("dq", "dk", "dv") if backward else ("o",)
    out = {x: torch.zeros(s[x].shape, dtype=torch.float64, device=DEV) for x in names}
    if not backward and case["train"]:
        out["lse"] = torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
    for i, (q0, lq, k0, lk) in enumerate(s["lengths"]):
        row = torch.arange(lq, device=DEV).unsqueeze(1) + lk - lq
        col = torch.arange(lk, device=DEV).unsqueeze(0)
        hidden = (col > row) | ((row - col >= case["window"]) & (col >= case["sinks"]))
        cut = lambda x, a, b, h: (s[x][a:a + b, h] if packed else s[x][i, a:a + b, h]).double()  # noqa: E731
        at = lambda a, b, h: (slice(a, a + b), h) if packed else (i, slice(a, a + b), h)  # noqa: E731
        for h in range(hq):
            g = h * hkv // hq
            q, k, v = cut("q", q0, lq, h), cut("k", k0, lk, g), cut("v", k0, lk, g)
            x = torch.einsum("id,jd->ij", q, k).mul_(s["scale"]).masked_fill_(hidden, -math.inf)
            if not backward:
                out["o"][at(q0, lq, h)] = torch.einsum("ij,jd->id", torch.softmax(x, -1).nan_to_num_(nan=0.0), v)
                if "lse" in out:
                    out["lse"][(h, slice(q0, q0 + lq)) if packed else (i, h)] = torch.logsumexp(x, -1)
                continue
            do, o = cut("do", q0, lq, h), cut("o", q0, lq, h)
            lse = (s["lse"][h, q0:q0 + lq] if packed else s["lse"][i, h]).double()
            p = torch.exp(x - lse[:, None]).masked_fill_(hidden, 0.0)
            ds = torch.einsum("id,jd->ij", do, v).sub_(torch.einsum("id,id->i", do, o)[:, None]).mul_(p)
            out["dq"][at(q0, lq, h)] = torch.einsum("ij,jd->id", ds, k) * s["scale"]
            out["dk"][at(k0, lk, g)] += torch.einsum("ij,id->jd", ds, q) * s["scale"]
            out["dv"][at(k0, lk, g)] += torch.einsum("ij,id->jd", p, do)
    return out


def _exact_rotary(s):
    case = s["case"]
    sections = _sections(case)
    half, out = sum(sections), {}
    turn = torch.empty((case["tokens"], half), dtype=torch.complex128, device=DEV)
    j = 0
    for a, n in enumerate(sections):
        for i in range(n):
            power = i / n if case["ladders"] else j / half
            angle = s["positions"][a].double() * math.exp(-math.log(10000.0) * power)
            turn[:, j] = torch.polar(torch.ones_like(angle), -angle if case["inverse"] else angle)
            j += 1
    for name in ("q", "k"):
        y = s[name].double().clone()
        even, odd = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["interleaved"] else (slice(0, half), slice(half, 2 * half))
        z = torch.complex(y[..., even].contiguous(), y[..., odd].contiguous()) * turn.unsqueeze(1)
        y[..., even], y[..., odd] = z.real, z.imag
        out[name] = y
    return out


def _exact_resnorm(s):
    case, d64 = s["case"], torch.float64
    layer, post, rows = case["kind"] == "layer", case["post"], case["rows"]
    wide = {k: v.to(d64) for k, v in s.items() if torch.is_tensor(v)}
    one = torch.ones(case["d"], dtype=d64, device=DEV)
    w1, w2, b1, b2 = wide.get("w1", one), wide["w2"], wide.get("b1", 0 * one), wide.get("b2", 0 * one)
    gate = torch.repeat_interleave(wide["gate"], case["gate_rows"], 0)[:rows] if "gate" in wide else one.expand(rows, -1)

    def moments(x):
        if layer:
            var, mean = torch.var_mean(x, dim=1, correction=0)
        else:
            var, mean = torch.linalg.vector_norm(x, dim=1).square() / x.shape[1], torch.zeros(rows, dtype=d64, device=DEV)
        return mean, torch.rsqrt(var + NORM_EPS)

    if case["op"] == "resnorm_fwd":
        out, n = {}, wide["y"]
        if post:
            mean, rstd = moments(n)
            n = torch.addcmul(b1, (n - mean[:, None]) * rstd[:, None], w1)
            out.update(rstd1=rstd, **({"mean1": mean} if layer else {}))
        z = torch.addcmul(wide["x"], n, gate, value=s["alpha"])
        mean, rstd = moments(z)
        u = torch.addcmul(b2, (z - mean[:, None]) * rstd[:, None], w2)
        return {**out, **({"mean2": mean} if layer else {}), "rstd2": rstd, "z": z, "u": u}

    def back(g, hat, rstd):
        r = g - hat * (g * hat).sum(1, keepdim=True) / case["d"]
        if layer:
            r -= g.sum(1, keepdim=True) / case["d"]
        return r * rstd[:, None]

    none = torch.zeros(rows, dtype=d64, device=DEV)
    hat2 = (wide["z"] - wide.get("mean2", none)[:, None]) * wide["rstd2"][:, None]
    t = wide["dz"] + back(wide["du"] * w2, hat2, wide["rstd2"])
    out = {"dx": t, "dw2": torch.einsum("rc,rc->c", wide["du"], hat2)}
    dn = s["alpha"] * gate * t
    n = wide["y"]
    if post:
        hat1 = (wide["y"] - wide.get("mean1", none)[:, None]) * wide["rstd1"][:, None]
        n = torch.addcmul(b1, hat1, w1)
        out["dy"] = back(dn * w1, hat1, wide["rstd1"])
        out["dw1"] = torch.einsum("rc,rc->c", dn, hat1)
    else:
        out["dy"] = dn
    if layer:
        out["db2"] = wide["du"].sum(0)
        if post:
            out["db1"] = dn.sum(0)
    if "gate" in wide:
        each = s["alpha"] * t * n
        out["dgate"] = torch.stack([part.sum(0) for part in each.split(case["gate_rows"])])
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("attn"):
        return _exact_attention(s)
    return _exact_rotary(s) if case["op"] == "rotary" else _exact_resnorm(s)
