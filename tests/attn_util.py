"""Rotation, attention and its gradients, and the 4-bit cache in 64 bits on the
CPU, with bounds on what a right kernel may be off, value by value.

Bounds count roundings.  HALF: half a step of the state dtype relative to the
value, for each rounding to it: outputs, and with a bf16 state the probabilities
and the gradients of scores, which are operands of the next product.  fp32
arithmetic: one 2^-24 an operation of the longest chain, so (K + a few) 2^-24 of
the sum of absolute products over K terms, whatever their order.  A score s
carries its product's error and some 2^-24 of its own size and of its row's
largest (it is taken relative to that); exp turns what it is off into a relative
error of the probability."""

import math

import torch

from tests.ffn_util import F64, HALF, U, assert_within  # noqa: F401


def spans(T, S, window=0, starts=None, prefix=None):
    """(lo, hi) of each token, token by token from the definitions."""
    lo, hi = [0] * T, [0] * T
    if starts is None:
        starts, prefix = list(range(0, T + 1, S)), None
    for i, (a, b) in enumerate(zip(starts, starts[1:])):
        for t in range(max(a, 0), min(b, T)):
            lo[t], hi[t] = max(a, 0), t + 1
            if prefix is not None:
                hi[t] = max(t + 1, min(a + prefix[i], b, T))
            if window:
                lo[t] = max(lo[t], t - window + 1)
    return torch.tensor(lo), torch.tensor(hi)


def rotated(x, cs, R, pairs, inverse=False):
    """x [T, heads, D] turned by cs [T, R / 2, 2], in fp32 as it is defined: each product and sum rounded."""
    x, cs = x.float(), cs.float()
    i = torch.arange(R // 2)
    a, b = (i, i + R // 2) if pairs == "halves" else (2 * i, 2 * i + 1)
    c, s = cs[:, None, :, 0], cs[:, None, :, 1] * (-1.0 if inverse else 1.0)
    y = x.clone()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


HELD = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=F64)


def held(x):
    """The values that the cache holds for x [.., D] (fp32), in 64 bits: by search of the nearest code."""
    y = x.float().reshape(*x.shape[:-1], -1, 32)
    top = y.abs().amax(-1, keepdim=True)
    scale = (top / 6.0).bfloat16().float()
    scale = torch.where(top < 2.0 ** -100, torch.zeros_like(scale), scale)
    scale = torch.where(torch.isfinite(top), scale, torch.full_like(scale, float("nan")))
    a = torch.where(scale > 0, y.abs() / torch.where(scale > 0, scale, torch.ones_like(scale)),
                    torch.zeros_like(y)).to(F64)                  # (the division is rounded to fp32)
    d = (a.unsqueeze(-1) - HELD).abs()
    near = d == d.amin(-1, keepdim=True)
    even = near & (torch.arange(8) % 2 == 0)
    pick = torch.where(even.any(-1, keepdim=True), even, near).to(torch.uint8).argmax(-1)
    v = torch.sign(y).to(F64) * HELD[pick] * scale.to(F64)
    return v.reshape(x.shape)


def scores(q, k, scale, cap, slope, dist):
    """Scores of one head, what they may be off, d score / d (scale q k) and what that may be off."""
    D = q.shape[1]
    x = q @ k.t() * scale
    ex = (D + 8) * U * (q.abs() @ k.abs().t()) * scale
    der, eder = torch.ones_like(x), torch.zeros_like(x)
    if cap:
        t = torch.tanh(x / cap)
        ex = ex + 16 * U * cap + 4 * U * x.abs()
        der, eder = 1 - t * t, 2 * ex / cap + 4 * U
        x = cap * t
    s = x - slope * dist
    return s, ex + 8 * U * (x.abs() + slope * dist), der, eder


def attention(q, k, v, seen, scale, cap, slope, dist, half, dout=None):
    """One head: dict of name -> (value, bound) for out and, given dout, dq, dk, dv; all in 64 bits."""
    n = k.shape[0]
    s, es, der, eder = scores(q, k, scale, cap, slope, dist)
    some = seen.any(1, keepdim=True)
    s = torch.where(seen, s, torch.full_like(s, -math.inf))
    top = torch.where(some, s.amax(1, keepdim=True), torch.zeros_like(s[:, :1]))
    es = torch.where(seen, es, torch.zeros_like(es)) + 8 * U * (top.abs() + torch.where(seen, s - top, 0 * es).abs())
    e = torch.where(seen, torch.exp(s - top), torch.zeros_like(s))
    sums = e.sum(1, keepdim=True)
    p = torch.where(some, e / sums.clamp(min=1e-300), e)
    worst = (es * seen).amax(1, keepdim=True) + (n + 16) * U
    out = p @ v
    eo = (p * (es + worst + half + (n + 16) * U)) @ v.abs()
    r = dict(out=(out, eo + half * (out.abs() + eo)))
    if dout is None:
        return r
    lse = torch.where(some, top + torch.log(sums.clamp(min=1e-300)), torch.zeros_like(top))
    ep = es + worst + 8 * U * (1 + lse.abs())
    eo = r["out"][1]
    D = q.shape[1]
    delta = (dout * out).sum(1, keepdim=True)
    edelta = (dout.abs() * eo).sum(1, keepdim=True) + (D + 8) * U * (dout.abs() * (out.abs() + eo)).sum(1, keepdim=True)
    dP = dout @ v.t()
    edP = (D + 8) * U * (dout.abs() @ v.abs().t())
    dS = p * (dP - delta) * der
    off = (dP - delta).abs()
    eS = p * (ep * (off + edP + edelta) + edP + edelta + 4 * U * off) * der.abs() + p * off * eder
    eS = eS + half * (dS.abs() + eS)
    T = q.shape[0]
    grow = lambda m, em, w, K: em @ w.abs() + (K + 8) * U * ((m.abs() + em) @ w.abs())   # noqa: E731
    dq, dk = scale * (dS @ k), scale * (dS.t() @ q)
    dv = p.t() @ dout
    r["dq"] = (dq, scale * grow(dS, eS, k, n) + 4 * U * dq.abs())
    r["dk"] = (dk, scale * grow(dS.t(), eS.t(), q, T) + 4 * U * dk.abs())
    r["dv"] = (dv, grow(p.t(), (p * (ep + half)).t(), dout, T))
    return r


def all_heads(qkv, lo, hi, Hq, Hkv, scale, cap=0.0, slopes=None, dout=None):
    """Every head's, as the tensors of a call: out, and with dout dqkv; (value, bound) each."""
    half, T = HALF[qkv.dtype], qkv.shape[0]
    x = qkv.cpu().to(F64)
    go = None if dout is None else dout.cpu().to(F64)
    j = torch.arange(T)
    seen = (j[None, :] >= lo[:, None]) & (j[None, :] < hi[:, None])
    dist = (j[:, None] - j[None, :]).abs().to(F64)
    out = [torch.zeros(T, Hq, x.shape[2], dtype=F64) for _ in range(2)]
    dx = [torch.zeros_like(x) for _ in range(2)]
    for h in range(Hq):
        kh = h // (Hq // Hkv)
        r = attention(x[:, h], x[:, Hq + kh], x[:, Hq + Hkv + kh], seen, scale, cap,
                      0.0 if slopes is None else float(slopes[h]), dist, half if half > U else 0.0,
                      None if go is None else go[:, h])
        for i in range(2):
            out[i][:, h] = r["out"][i]
            if go is not None:
                for at, n in ((h, "dq"), (Hq + kh, "dk"), (Hq + Hkv + kh, "dv")):
                    dx[i][:, at] += r[n][i]
    if half == U:
        out[1] += U * out[0].abs()
    dx[1] += (Hq // Hkv + 4) * U * dx[0].abs() + half * (dx[0].abs() + dx[1])
    return tuple(out), tuple(dx)


def inputs(T, Hq, Hkv, D, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, Hq + 2 * Hkv, D, generator=g).to(dtype), torch.randn(T, Hq, D, generator=g).to(dtype))
