"""Cases that measure the training operators: AdamW over a list of tensors (with the clip factor from the gradients'
norm, states in 32 or 8 bits), layer norm and the gated feed-forward block, each forward and backward.

``run`` computes them in plain torch operations, or, where ``own`` is set, with this package's kernels.
"""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 256                       # elements that share a scale in the 8-bit states; tensors start at multiples of it
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
HYPER = {"lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.01}
LN_EPS = 1e-5
SMALLEST = 2.0 ** -100            # a block whose largest state is below this is held as zeros
MASK32 = 0xFFFFFFFF


# ----------------------------------------------------------------- the cases
def listed():
    return [
        # one optimiser step of a small model held as one flat vector: launch latency
        {"name": "adamw32_flat_1m", "op": "adamw", "bits": 32, "layout": "ragged", "tensors": 1, "total": 1 << 20,
         "grad": "f32", "copy": False, "clip": True, "skew": 0},
        # the whole 48-layer transformer of the benchmark, 580 tensors, fp32 gradients, clipped
        {"name": "adamw32_gpt2_xl", "op": "adamw", "bits": 32, "layout": "transformer", "layers": 48, "d": 1600,
         "vocab": 50257, "positions": 1024, "grad": "f32", "copy": False, "clip": True, "skew": 0},
        # a convolutional network's list of 161 tensors from one element to millions, at odd addresses
        {"name": "adamw8_161_tensors", "op": "adamw", "bits": 8, "layout": "ragged", "tensors": 161, "total": 25_557_032,
         "grad": "bf16", "copy": False, "clip": False, "skew": 1},
        # a pipeline stage of eight blocks in mixed precision: 16-bit gradients, 16-bit copy of the weights written
        {"name": "adamw8_8_blocks", "op": "adamw", "bits": 8, "layout": "transformer", "layers": 8, "d": 1600,
         "vocab": 0, "positions": 0, "grad": "bf16", "copy": True, "clip": False, "skew": 0},
        # a handful of tokens: latency
        {"name": "ln_fwd_16x1600", "op": "ln_fwd", "rows": 16, "d": 1600, "dtype": "bf16", "param": "f32", "pad": 0},
        # a full batch of 64 sequences of 1024 tokens
        {"name": "ln_fwd_65536x1600", "op": "ln_fwd", "rows": 65536, "d": 1600, "dtype": "bf16", "param": "f32", "pad": 0},
        # fp32 rows of odd length inside a wider buffer
        {"name": "ln_bwd_2047x1001", "op": "ln_bwd", "rows": 2047, "d": 1001, "dtype": "f32", "param": "f32", "pad": 7},
        {"name": "ln_bwd_65536x1600", "op": "ln_bwd", "rows": 65536, "d": 1600, "dtype": "bf16", "param": "bf16", "pad": 0},
        # one token through the block of the benchmark's width: the weights' bytes count
        {"name": "ffn_fwd_1x1600x6400", "op": "ffn_fwd", "tokens": 1, "d": 1600, "f": 6400, "dtype": "bf16",
         "act": "silu", "train": False, "pad": 0},
        # a training batch's forward pass, with what the backward pass needs
        {"name": "ffn_fwd_8192x1600x6400", "op": "ffn_fwd", "tokens": 8192, "d": 1600, "f": 6400, "dtype": "bf16",
         "act": "silu", "train": True, "pad": 0},
        # odd width and hidden size, rows that start at odd addresses
        {"name": "ffn_bwd_1000x777x2051", "op": "ffn_bwd", "tokens": 1000, "d": 777, "f": 2051, "dtype": "f16",
         "act": "gelu_tanh", "pad": 0},
        {"name": "ffn_bwd_8192x1600x6400", "op": "ffn_bwd", "tokens": 8192, "d": 1600, "f": 6400, "dtype": "bf16",
         "act": "silu", "pad": 0},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _width(rng, lo, hi):
    """A row length: most often a multiple of 8, as in models, else any."""
    n = _log_int(rng, lo, hi)
    if rng.random() < 0.7:
        n = max(8, n // 8 * 8)
    return n + 8 if n == 3 << 10 else n


def draw(rng):
    op = rng.choice(["adamw", "adamw", "ln_fwd", "ln_bwd", "ffn_fwd", "ffn_bwd"])
    if op == "adamw":
        total = _log_int(rng, 1000, 300_000_000)
        bits = rng.choice([8, 32])
        return {"op": op, "bits": bits, "layout": "ragged", "tensors": _log_int(rng, 1, min(600, total // 20)), "total": total,
                "grad": rng.choice(["f32", "bf16", "f16"]), "copy": rng.random() < 0.4,
                "clip": bits == 32 and rng.random() < 0.6, "skew": rng.choice([0, 0, 1, 4])}
    if op.startswith("ln"):
        d = _width(rng, 16, 16384)
        rows = _log_int(rng, 1, min(65536, 65536 * 1600 // d))
        dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
        return {"op": op, "rows": rows, "d": d, "dtype": dtype, "param": rng.choice(["f32", dtype]),
                "pad": rng.choice([0, 0, 8, 3])}
    d, f = _width(rng, 64, 4096), _width(rng, 64, 8192)
    case = {"op": op, "tokens": _log_int(rng, 1, 8192), "d": d, "f": f, "dtype": rng.choice(["bf16", "bf16", "f16"]),
            "act": rng.choice(["silu", "silu", "gelu_tanh"]), "pad": rng.choice([0, 0, 8, 3])}
    if op == "ffn_fwd":
        case["train"] = rng.random() < 0.5
    return case


def _numel(case):
    """Element counts of the case's tensors."""
    if case["layout"] == "transformer":
        d = case["d"]
        one = [d, d, 3 * d * d, 3 * d, d * d, d, d, d, 4 * d * d, 4 * d, 4 * d * d, d]
        head = [case["vocab"] * d, case["positions"] * d] if case["vocab"] else []
        return head + one * case["layers"] + [d, d]
    n, total = case["tensors"], case["total"]
    if n == 1:
        return [total]
    # sizes spread over four decades, from one element up, adding up to the total
    weight = [10.0 ** (4.0 * ((i * 0.6180339887498949) % 1.0)) for i in range(n)]
    size = [max(1, int(total * x / sum(weight))) for x in weight]
    big = max(range(n), key=size.__getitem__)
    size[big] += total - sum(size)
    return [max(1, x) for x in size]


def _starts(numel):
    """Where each tensor starts in the flat state buffers, and their length: every tensor begins a new block."""
    at, starts = 0, []
    for n in numel:
        starts.append(at)
        at += -(-n // BLOCK) * BLOCK
    return starts, at


# ----------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(DEV).manual_seed(int(seed) % (1 << 62))


def _normal(gen, *shape, std=1.0):
    return torch.empty(shape, device=DEV).normal_(0.0, std, generator=gen)


def _rows(values, dtype, pad):
    """The values as rows of a buffer that is ``pad`` elements wider."""
    r, c = values.shape
    buf = torch.zeros((r, c + pad), dtype=dtype, device=DEV)
    buf[:, :c].copy_(values)
    return buf[:, :c]


def _empty_rows(r, c, dtype, pad):
    return torch.zeros((r, c + pad), dtype=dtype, device=DEV)[:, :c]


def _prepare_adamw(case, seed):
    gen, numel = _gen(seed), _numel(case)
    starts, n = _starts(numel)
    skew, eight = case["skew"], case["bits"] == 8
    wide = lambda dtype: torch.zeros(n + skew, dtype=dtype, device=DEV)[skew:]  # noqa: E731
    w, g = wide(torch.float32), wide(DTYPES[case["grad"]])
    copy = wide(torch.bfloat16) if case["copy"] else None
    rms = torch.zeros(n, device=DEV)          # the scale of each tensor's gradients, zero between tensors
    scales = (10.0 ** torch.empty(len(numel)).uniform_(-4.0, -2.0, generator=torch.Generator().manual_seed(int(seed) % (1 << 62)))).tolist()
    for at, k, s in zip(starts, numel, scales):
        rms[at:at + k] = s
    w.copy_(_normal(gen, n, std=0.02)).mul_(rms > 0)
    g.copy_(_normal(gen, n).mul_(rms))
    m = _normal(gen, n, std=0.3).mul_(rms)
    r = _normal(gen, n, std=0.25).exp_().mul_(rms)
    del rms
    s = {"case": case, "w": w, "g": g, "copy": copy, "t": 100, "norm": torch.zeros(2, device=DEV)}
    if eight:
        m, r = m.view(-1, BLOCK), r.view(-1, BLOCK)
        am, ar = m.abs().amax(1), r.amax(1)
        s["m"] = (m.div(am[:, None].clamp_min(1e-30)).abs_().sqrt_().mul_(127.0).round_() * m.sign()).to(torch.int8).view(-1)
        s["v"] = r.div(ar[:, None].clamp_min(1e-30)).sqrt_().mul_(255.0).round_().clamp_min_(2.0).to(torch.uint8).view(-1)
        s["ms"], s["vs"] = am, ar
        s["m_out"], s["v_out"] = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    else:
        s["m"], s["v"] = m, r.mul_(r)
    cut = lambda flat: [flat[at:at + k] for at, k in zip(starts, numel)]  # noqa: E731
    s["ws"], s["gs"], s["copies"] = cut(w), cut(g), cut(copy) if copy is not None else None
    if own:
        from paper_2006_07405_b200 import binding as B
        s["B"] = B
        s["plan"] = B.a2sgd_adamw_create(s["ws"], s["gs"], s["m"], s["v"], m_scale=s.get("ms"), v_scale=s.get("vs"),
                                         w16=s["copies"])
    return s


def _prepare_ln(case, seed):
    gen = _gen(seed)
    rows, d, dtype, param, pad = case["rows"], case["d"], DTYPES[case["dtype"]], DTYPES[case["param"]], case["pad"]
    x = _normal(gen, rows, d) * _normal(gen, rows, 1, std=0.5).exp_() + _normal(gen, 1, d, std=0.5)
    s = {"case": case, "x": _rows(x, dtype, pad), "w": (1.0 + _normal(gen, d, std=0.2)).to(param),
         "b": _normal(gen, d, std=0.2).to(param)}
    if case["op"] == "ln_fwd":
        s.update(y=_empty_rows(rows, d, dtype, pad), mean=torch.empty(rows, device=DEV), rstd=torch.empty(rows, device=DEV))
    else:
        x = s["x"].float()
        mean = x.mean(1)
        rstd = ((x - mean[:, None]).square().mean(1) + LN_EPS).rsqrt()
        s.update(dy=_rows(_normal(gen, rows, d), dtype, pad), mean=mean, rstd=rstd, dx=_empty_rows(rows, d, dtype, pad),
                 dw=torch.empty(d, dtype=param, device=DEV), db=torch.empty(d, dtype=param, device=DEV))
    if own:
        from paper_2006_07405_b200 import binding as B
        s["B"] = B
        if case["op"] == "ln_bwd":
            s["work"] = torch.empty(B.a2sgd_layer_norm_workspace(rows, d), dtype=torch.uint8, device=DEV)
    return s


def _prepare_ffn(case, seed):
    gen = _gen(seed)
    t, d, f, dtype, pad = case["tokens"], case["d"], case["f"], DTYPES[case["dtype"]], case["pad"]
    s = {"case": case, "x": _rows(_normal(gen, t, d), dtype, pad), "wg": _rows(_normal(gen, f, d, std=d ** -0.5), dtype, pad),
         "wu": _rows(_normal(gen, f, d, std=d ** -0.5), dtype, pad), "wd": _rows(_normal(gen, d, f, std=f ** -0.5), dtype, pad)}
    rows = lambda r, c: _empty_rows(r, c, dtype, pad)  # noqa: E731
    if case["op"] == "ffn_fwd":
        s.update(y=rows(t, d), h=rows(t, f), a=rows(t, f) if case["train"] else None, b=rows(t, f) if case["train"] else None)
    else:
        # what the forward pass of this step left behind
        a, b = s["x"].float() @ s["wg"].float().T, s["x"].float() @ s["wu"].float().T
        s["a"], s["b"] = _rows(a, dtype, pad), _rows(b, dtype, pad)
        s["h"] = _rows(_act(a, case["act"])[0] * b, dtype, pad)
        s.update(dy=_rows(_normal(gen, t, d), dtype, pad), dx=rows(t, d), dwg=rows(f, d), dwu=rows(f, d), dwd=rows(d, f))
    if own:
        from paper_2006_07405_b200 import binding as B
        s["B"] = B
        s["work"] = torch.empty(B.a2sgd_gated_ffn_workspace(t, d, f, backward=case["op"] == "ffn_bwd"), dtype=torch.uint8, device=DEV)
    return s


def prepare(case, seed):
    if case["op"] == "adamw":
        return _prepare_adamw(case, seed)
    return _prepare_ln(case, seed) if case["op"].startswith("ln") else _prepare_ffn(case, seed)


# ----------------------------------------------------------------- the plain forms
def _dither(n, step):
    """Two 12-bit numbers for each element of the state from a counter hash of the step and the element's place."""
    h = torch.arange(n, device=DEV) * 0x9E3779B1 + ((step * 0x85A308D3 + 0x243F6A89) & MASK32)
    h &= MASK32
    h ^= h >> 16
    h = (h * 0x7FEB3525) & MASK32
    h ^= h >> 15
    h = (h * 0x94D049BB) & MASK32
    h ^= h >> 16
    return h >> 20, (h >> 8) & 0xFFF


def _encode(x, top, dither):
    """Codes 0..127 or 0..255 and the scale of each row of non-negative values: x is about (q / qmax)^2 * scale, rounded up
    or down by the dither so that the expectation is x. ``top`` is qmax."""
    scale = x.amax(1, keepdim=True)
    scale = torch.where(scale < SMALLEST, torch.zeros_like(scale), scale)
    gain = torch.where(scale > 0, float(top * top) / scale, torch.zeros_like(scale))
    s = x * gain
    q = s.sqrt().floor()
    q = q + (s - q * q > dither.view(x.shape).float() * (1.0 / 4096.0) * (2.0 * q + 1.0))
    return q.clamp(max=float(top)), scale


def _adamw_constants(t):
    h = HYPER
    return {"decay": 1.0 - h["lr"] * h["weight_decay"], "rate": h["lr"] / (1.0 - h["beta1"] ** t),
            "root": 1.0 / math.sqrt(1.0 - h["beta2"] ** t)}


def _plain_adamw(s):
    case, h = s["case"], HYPER
    s["t"] += 1
    k, eight = _adamw_constants(s["t"]), case["bits"] == 8
    g = s["g"].float()
    if case["clip"]:
        norm = (g * g).sum().sqrt()
        scale = 1.0 / norm.clamp(min=1.0)       # norm clipped to 1
        s["norm"].copy_(torch.stack([norm, scale]))
        g = g * scale
    if eight:
        q, am, ar = s["m"].float().view(-1, BLOCK), s["ms"][:, None], s["vs"][:, None]
        m = ((q * q.abs()) * (am / 16129.0)).view(-1)
        q = s["v"].float().view(-1, BLOCK)
        r = ((q * q) * (ar / 65025.0)).view(-1)
        v = r * r
    else:
        m, v = s["m"], s["v"]
    m = m * h["beta1"] + g * (1.0 - h["beta1"])
    v = v * h["beta2"] + (g * g) * (1.0 - h["beta2"])
    r = v.sqrt()
    w = s["w"]
    w.copy_(w * k["decay"] - (m / (r * k["root"] + h["eps"])) * k["rate"])
    out = {"w": w}
    if s["copy"] is not None:
        out["copy"] = s["copy"].copy_(w)
    if case["clip"]:
        out["norm"] = s["norm"]
    if not eight:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return {**out, "m": s["m"], "v": s["v"]}
    um, ur = _dither(m.numel(), s["t"])
    m, r = m.view(-1, BLOCK), r.view(-1, BLOCK)
    q, am = _encode(m.abs(), 127, um)
    q = torch.where(m < 0, -q, q)
    s["m"].copy_(q.view(-1))
    s["ms"].copy_(am.view(-1))
    s["m_out"].copy_(((q * q.abs()) * (am / 16129.0)).view(-1))
    q, ar = _encode(r, 255, ur)
    q = q.clamp(min=2.0)
    s["v"].copy_(q.view(-1))
    s["vs"].copy_(ar.view(-1))
    r = ((q * q) * (ar / 65025.0)).view(-1)
    s["v_out"].copy_(r * r)
    return {**out, "m": s["m_out"], "v": s["v_out"]}


def _plain_ln_fwd(s):
    x, d = s["x"].float(), s["case"]["d"]
    mean = x.sum(1, keepdim=True) * (1.0 / d)
    c = x - mean
    rstd = 1.0 / ((c * c).sum(1, keepdim=True) * (1.0 / d) + LN_EPS).sqrt()
    y = (c * rstd * s["w"].float() + s["b"].float()).to(s["x"].dtype)
    return {"y": y, "mean": mean.view(-1), "rstd": rstd.view(-1)}


def _plain_ln_bwd(s):
    x, dy, d = s["x"].float(), s["dy"].float(), s["case"]["d"]
    rstd = s["rstd"][:, None]
    xhat = (x - s["mean"][:, None]) * rstd
    g = dy * s["w"].float()
    dx = (g - g.sum(1, keepdim=True) * (1.0 / d) - xhat * ((g * xhat).sum(1, keepdim=True) * (1.0 / d))) * rstd
    return {"dx": dx.to(s["x"].dtype), "dw": (dy * xhat).sum(0).to(s["w"].dtype), "db": dy.sum(0).to(s["w"].dtype)}


def _act(a, name):
    """The activation and its derivative."""
    if name == "silu":
        p = 1.0 / (1.0 + (-a).exp())
        return a * p, p * (1.0 + a * (1.0 - p))
    k, c = 2.0 * math.sqrt(2.0 / math.pi), 0.044715
    p = 1.0 / (1.0 + (-(k * (a + c * a * a * a))).exp())
    return a * p, p + a * p * (1.0 - p) * (k * (1.0 + 3.0 * c * a * a))


def _plain_ffn_fwd(s):
    x, dtype = s["x"].float(), s["x"].dtype
    a, b = x @ s["wg"].float().T, x @ s["wu"].float().T
    h = _act(a, s["case"]["act"])[0] * b
    out = {"y": (h @ s["wd"].float().T).to(dtype)}
    if s["case"]["train"]:
        out.update(a=a.to(dtype), b=b.to(dtype), h=h.to(dtype))
    return out


def _plain_ffn_bwd(s):
    dy, x, a, b, h = (s[k].float() for k in ("dy", "x", "a", "b", "h"))
    dtype = s["x"].dtype
    act, slope = _act(a, s["case"]["act"])
    dh = dy @ s["wd"].float()
    da, db = dh * b * slope, dh * act
    return {"dx": (da @ s["wg"].float() + db @ s["wu"].float()).to(dtype), "dwg": (da.T @ x).to(dtype),
            "dwu": (db.T @ x).to(dtype), "dwd": (dy.T @ h).to(dtype)}


# ----------------------------------------------------------------- the framework's calls
def _own_adamw(s):
    B, case = s["B"], s["case"]
    s["t"] += 1
    out = {"w": s["w"]}
    if case["clip"]:
        B.a2sgd_adamw_grad_norm(s["plan"], 1.0, s["norm"])
        out["norm"] = s["norm"]
    B.a2sgd_adamw_step(s["plan"], step=s["t"], grad_scale=s["norm"][1:] if case["clip"] else None, **HYPER)
    if s["copy"] is not None:
        out["copy"] = s["copy"]
    if case["bits"] == 32:
        return {**out, "m": s["m"], "v": s["v"]}
    B.a2sgd_adamw_read_state(s["plan"], s["m_out"], s["v_out"])
    return {**out, "m": s["m_out"], "v": s["v_out"]}


def _own_ln_fwd(s):
    s["B"].a2sgd_layer_norm_forward(s["x"], s["w"], s["b"], s["y"], s["mean"], s["rstd"], LN_EPS)
    return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}


def _own_ln_bwd(s):
    s["B"].a2sgd_layer_norm_backward(s["dy"], s["x"], s["w"], s["mean"], s["rstd"], s["dx"], s["dw"], s["db"], s["work"])
    return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}


def _own_ffn_fwd(s):
    s["B"].a2sgd_gated_ffn_forward(s["x"], s["wg"], s["wu"], s["wd"], s["y"], s["h"], s["a"], s["b"],
                                   activation=s["case"]["act"], workspace=s["work"])
    return {"y": s["y"], "a": s["a"], "b": s["b"], "h": s["h"]} if s["case"]["train"] else {"y": s["y"]}


def _own_ffn_bwd(s):
    s["B"].a2sgd_gated_ffn_backward(s["dy"], s["x"], s["wg"], s["wu"], s["wd"], s["h"], s["a"], s["b"],
                                    s["dx"], s["dwg"], s["dwu"], s["dwd"], activation=s["case"]["act"], workspace=s["work"])
    return {"dx": s["dx"], "dwg": s["dwg"], "dwu": s["dwu"], "dwd": s["dwd"]}


def run(state):
    op = state["case"]["op"]
    if own:
        return {"adamw": _own_adamw, "ln_fwd": _own_ln_fwd, "ln_bwd": _own_ln_bwd, "ffn_fwd": _own_ffn_fwd,
                "ffn_bwd": _own_ffn_bwd}[op](state)
    return {"adamw": _plain_adamw, "ln_fwd": _plain_ln_fwd, "ln_bwd": _plain_ln_bwd, "ffn_fwd": _plain_ffn_fwd,
            "ffn_bwd": _plain_ffn_bwd}[op](state)


# ----------------------------------------------------------------- the work
def work(case):
    op = case["op"]
    if op == "adamw":
        n, e = sum(_numel(case)), SIZES[case["grad"]]
        state = 16 if case["bits"] == 32 else 4 + 8 + 16 / BLOCK     # 8 bits: codes in and out, and the values they stand for
        return {"bytes": n * (8 + e + state + (2 if case["copy"] else 0)), "flops": 16 * n + (2 * n if case["clip"] else 0)}
    if op.startswith("ln"):
        rows, d, e, p = case["rows"], case["d"], SIZES[case["dtype"]], SIZES[case["param"]]
        tensors, vectors = (2, 2) if op == "ln_fwd" else (3, 3)
        return {"bytes": tensors * rows * d * e + vectors * d * p + 8 * rows, "flops": (8 if op == "ln_fwd" else 14) * rows * d}
    t, d, f, e = case["tokens"], case["d"], case["f"], SIZES[case["dtype"]]
    if op == "ffn_fwd":
        return {"bytes": e * (3 * d * f + 2 * t * d + (3 * t * f if case["train"] else 0)), "flops": 6 * t * d * f}
    return {"bytes": e * (6 * d * f + 3 * t * d + 3 * t * f), "flops": 12 * t * d * f}


# ----------------------------------------------------------------- the definition in 64 bits
def _exact_codes(x, top, u):
    """q and the scale of rows of non-negative values in 64 bits."""
    scale = x.max(dim=1, keepdim=True).values
    scale[scale < SMALLEST] = 0.0
    s = torch.nan_to_num(x * (top ** 2 / scale), nan=0.0, posinf=0.0)
    q = torch.trunc(torch.pow(s, 0.5))
    up = (s - q ** 2) * 4096.0 > u.reshape(x.shape) * (2.0 * q + 1.0)
    return torch.minimum(q + up, torch.full_like(q, float(top))), scale


def _exact_adamw(s):
    case, d64 = s["case"], torch.float64
    t = s["t"] + 1
    lr, b1, b2, eps, wd = (HYPER[k] for k in ("lr", "beta1", "beta2", "eps", "weight_decay"))
    eight = case["bits"] == 8
    g, out = s.pop("g").to(d64), {}
    s["gs"] = None
    if case["clip"]:
        norm = torch.linalg.vector_norm(g)
        scale = torch.clamp(1.0 / norm, max=1.0)
        out["norm"] = torch.stack([norm, scale])
        g *= scale
    if eight:
        code = s["m"].to(d64)
        m = torch.copysign(code.square(), code).view(-1, BLOCK).mul_(s["ms"].to(d64)[:, None] / 127 ** 2).view(-1)
        v = (s["v"].to(d64) / 255).pow(2).view(-1, BLOCK).mul_(s["vs"].to(d64)[:, None]).pow_(2).view(-1)
    else:
        m, v = s.pop("m").to(d64), s.pop("v").to(d64)
    m.lerp_(g, 1.0 - b1)
    v.mul_(b2).addcmul_(g, g, value=1.0 - b2)
    del g
    w = s.pop("w").to(d64)
    s["ws"] = None
    w.mul_(1.0 - lr * wd).addcdiv_(m, (v / (1.0 - b2 ** t)).sqrt_().add_(eps), value=-lr / (1.0 - b1 ** t))
    out["w"] = w
    if case["copy"]:
        out["copy"] = w
    if eight:
        um, ur = _dither(m.numel(), t)
        q, scale = _exact_codes(m.abs().view(-1, BLOCK), 127, um)
        m = (q.pow(2) * scale / 127 ** 2).view(-1).copysign(m)
        q, scale = _exact_codes(v.sqrt().view(-1, BLOCK), 255, ur)
        v = (q.clamp_(min=2.0).pow(2) * scale / 255 ** 2).pow(2).view(-1)
    return {**out, "m": m, "v": v}


def _exact_ln(s):
    x, w, b = s["x"].double(), s["w"].double(), s["b"].double()
    if s["case"]["op"] == "ln_fwd":
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = (var + LN_EPS).pow(-0.5)
        return {"y": torch.addcmul(b, (x - mean[:, None]) * rstd[:, None], w), "mean": mean, "rstd": rstd}
    rstd, dy = s["rstd"].double()[:, None], s["dy"].double()
    z = (x - s["mean"].double()[:, None]) * rstd
    u = dy * w
    return {"dx": rstd * (u - u.mean(1, keepdim=True) - z * (u * z).mean(1, keepdim=True)),
            "dw": torch.einsum("rc,rc->c", dy, z), "db": dy.sum(0)}


def _exact_act(a, name):
    if name == "silu":
        p = torch.sigmoid(a)
        return p * a, p + p * (1 - p) * a
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (a + 0.044715 * a ** 3))
    return 0.5 * a * (1 + t), 0.5 * (1 + t) + 0.5 * a * (1 - t * t) * k * (1 + 3 * 0.044715 * a ** 2)


def _exact_ffn(s):
    act = s["case"]["act"]
    x, wg, wu, wd = (s[k].double() for k in ("x", "wg", "wu", "wd"))
    if s["case"]["op"] == "ffn_fwd":
        a, b = torch.einsum("td,fd->tf", x, wg), torch.einsum("td,fd->tf", x, wu)
        h = _exact_act(a, act)[0] * b
        out = {"y": torch.einsum("tf,df->td", h, wd)}
        return {**out, "a": a, "b": b, "h": h} if s["case"]["train"] else out
    dy, a, b, h = (s[k].double() for k in ("dy", "a", "b", "h"))
    value, slope = _exact_act(a, act)
    dh = torch.einsum("td,df->tf", dy, wd)
    da, db = slope * b * dh, value * dh
    return {"dx": torch.einsum("tf,fd->td", da, wg).add_(torch.einsum("tf,fd->td", db, wu)),
            "dwg": torch.einsum("tf,td->fd", da, x), "dwu": torch.einsum("tf,td->fd", db, x),
            "dwd": torch.einsum("td,tf->df", dy, h)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(s)
    return _exact_ln(s) if case["op"].startswith("ln") else _exact_ffn(s)
