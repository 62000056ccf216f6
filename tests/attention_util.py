"""The attention's definition in 64 bits, with the bound on what a kernel may be off by, for the tests."""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
F32 = 2.0 ** -24


def visible(lq, lk, window, sinks, device):
    place = torch.arange(lq, device=device)[:, None] + (lk - lq)
    key = torch.arange(lk, device=device)[None, :]
    return (key <= place) & ((key > place - window) | (key < sinks))


def reference(q, k, v, window, sinks, scale, dout=None, o=None, lse=None):
    """One sequence: q [lq, hq, d], k, v [lk, hkv, d] of a 16-bit type.  Returns {name: (value, bound)}.

    Bounds.  A score is a sum of d products in fp32, scaled: off by at most e = (d + 3) 2^-24 scale sum |q k|.  P is exp of
    score - maximum in fp32 through exp2 of a scaled argument (the scaled score is rounded: 2^-24 of itself and of the maximum, and the
    special function's 2^-22), so its relative error is at most r = 2 e + 2^-22 + 2^-22 (1 + |maximum|); it is then rounded to the 16-bit type:
    half a step h (the sum of the row takes P as it was).  P is at least 2^-14 of its row's scale where float16 keeps half a step, and
    off by 2^-25 absolutely below: 2^-24 sum |v| covers it.  Sums of up to 2^16 terms in blocks add 2^-16 at most of their absolute
    terms (fp32 accumulation of n terms in any order: n 2^-24).
    """
    u = HALF_STEP[q.dtype]
    lq, hq, d = q.shape
    lk, hkv = k.shape[:2]
    seen = visible(lq, lk, window, sinks, q.device)
    out = {n: (torch.zeros((r, h, d), dtype=torch.float64, device=q.device), torch.zeros((r, h, d), dtype=torch.float64, device=q.device))
           for n, r, h in (("o", lq, hq), ("dq", lq, hq), ("dk", lk, hkv), ("dv", lk, hkv))}
    out["lse"] = (torch.full((hq, lq), -math.inf, dtype=torch.float64, device=q.device), torch.zeros((hq, lq), dtype=torch.float64, device=q.device))
    terms = max(16, lq * (hq // hkv), lk) * F32
    for h in range(hq):
        g = h // (hq // hkv)
        qq, kk, vv = q[:, h].double(), k[:, g].double(), v[:, g].double()
        x = (qq @ kk.T * scale).masked_fill(~seen, -math.inf)
        most = (qq.abs() @ kk.abs().T * scale).masked_fill(~seen, 0.0)
        e = (d + 3) * F32 * (most.amax(1, keepdim=True) if lk else most.sum(1, keepdim=True))
        if dout is None:
            top = x.amax(1, keepdim=True).nan_to_num(neginf=0.0) if lk else torch.zeros_like(e)
            r = 2 * e + 2.0 ** -21 * (2 + top.abs())
            p = torch.exp(x - top)
            total = p.sum(1, keepdim=True)
            safe = torch.where(total > 0, total, torch.ones_like(total))
            a = p @ vv.abs() / safe
            value = p @ vv / safe
            out["o"][0][:, h], out["o"][1][:, h] = value, (u + 2 * r + terms) * a + u * value.abs() + 2.0 ** -24 * (seen.double() @ vv.abs()) / safe + 2.0 ** -24
            out["lse"][0][h], out["lse"][1][h] = (total.log() + top)[:, 0], (r + terms + 2.0 ** -21 * (1 + top.abs() + total.log().abs().nan_to_num(posinf=0.0)))[:, 0]
            continue
        dd, oo, ll = dout[:, h].double(), o[:, h].double(), lse[h].double()[:, None]
        p = torch.exp(x - ll).masked_fill(~seen, 0.0)
        r = 2 * e + 2.0 ** -21 * (2 + ll.abs().nan_to_num(posinf=0.0))
        dp = dd @ vv.T
        delta = (dd * oo).sum(1, keepdim=True)
        ds = p * (dp - delta)
        loose = (d + 3) * F32 * (dd.abs() @ vv.abs().T + (dd * oo).abs().sum(1, keepdim=True))   # of dp - delta
        off = (u + r + terms) * ds.abs() + p * loose + 2.0 ** -25 * seen
        out["dq"][0][:, h] = scale * ds @ kk
        out["dq"][1][:, h] = scale * off @ kk.abs() + terms * scale * ds.abs() @ kk.abs() + u * out["dq"][0][:, h].abs() + 2.0 ** -24
        out["dk"][0][:, g] += scale * ds.T @ qq
        out["dk"][1][:, g] += scale * (off + terms * ds.abs()).T @ qq.abs()
        out["dv"][0][:, g] += p.T @ dd
        out["dv"][1][:, g] += ((u + r + terms) * p + 2.0 ** -25 * seen).T @ dd.abs()
    for n in ("dk", "dv"):
        out[n][1].add_(u * out[n][0].abs() + 2.0 ** -24)
    return out


def check(name, got, value, bound):
    got = got.double()
    assert torch.equal(torch.isneginf(got), torch.isneginf(value)), f"{name}: other rows are empty"
    live = ~torch.isneginf(value)
    over = ((got - value).abs() - bound)[live]
    assert not torch.isnan(over).any(), f"{name}: not a number"
    assert over.numel() == 0 or over.max().item() <= 0.0, f"{name}: off by {(got - value).abs()[live].max().item()}, {over.max().item()} beyond its bound"
