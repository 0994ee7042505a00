"""The norm, the gated feed-forward block and the gradient clip in 64 bits on
the CPU, with bounds on what a right kernel may be off, value by value.

Bounds count roundings: HALF = half a step of the state dtype relative to the
value for each rounding to it (outputs; with a bf16 state also h, dg and du),
2^-15 for the saved g and u of a bf16 state (16 of their 24 significant bits
are kept, the rest is cut off), and for fp32 arithmetic one 2^-24 per operation of the
longest chain, i.e. (K + a few) 2^-24 of the sum of absolute products over K
terms, whatever their order."""

import math

import torch

F64 = torch.float64
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
U = 2.0 ** -24
# exp is good to about (3 + |its argument|) 2^-24, erf to a few 2^-24 of 1; arguments here are below 30
ACT = 64 * U
# largest |act'| and |act''|: SiLU 1.0999 (at 2.4) and 0.5 (at 0); GELU 1.129 (at sqrt 2) and 0.798 (at 0)
L1, L2 = 1.13, 0.8


def act(g, kind):
    if kind == "silu":
        e = torch.sigmoid(g)
        return g * e, e * (1 + g * (1 - e))
    e = 0.5 * torch.erfc(-g / math.sqrt(2.0))
    return g * e, e + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)


def ffn_forward(x, w, kind, half):
    """Values and bounds: dict of name -> (value, bound)."""
    x = x.to(F64)
    Wg, Wu, Wd = (w[n].bfloat16().to(F64) for n in ("W_gate", "W_up", "W_down"))
    C, H = Wg.shape
    g, u = x @ Wg, x @ Wu
    eg, eu = (C + 4) * U * (x.abs() @ Wg.abs()), (C + 4) * U * (x.abs() @ Wu.abs())
    a, da = act(g, kind)
    h = a * u
    eh = (L1 * eg + ACT * g.abs()) * (u.abs() + eu) + a.abs() * eu
    rounded = eh + half * (h.abs() + eh) if half > U else eh + U * h.abs()
    F = h @ Wd
    eF = rounded @ Wd.abs() + (H + 4) * U * ((h.abs() + rounded) @ Wd.abs())
    eF = eF + half * (F.abs() + eF)
    return dict(g=(g, eg), u=(u, eu), h=(h, rounded), F=(F, eF), a=a, da=da, W=(Wg, Wu, Wd))


def ffn_backward(x, dF, fw, kind, half):
    """Values and bounds of dx and the weight gradients, fw = ffn_forward's answer."""
    x, dF = x.to(F64), dF.to(F64)
    Wg, Wu, Wd = fw["W"]
    (g, eg), (u, eu) = fw["g"], fw["u"]
    C, H = Wg.shape
    T = x.shape[0]
    save = 2.0 ** -15 if half > U else 0.0
    eg, eu = eg + save * (g.abs() + eg), eu + save * (u.abs() + eu)
    a, da = fw["a"], fw["da"]
    dh = dF @ Wd.t()
    edh = (C + 4) * U * (dF.abs() @ Wd.abs().t())
    ea, eda = L1 * eg + ACT * g.abs(), L2 * eg + ACT * (1 + g.abs())
    h, du, dg = a * u, dh * a, dh * u * da
    eh = ea * (u.abs() + eu) + a.abs() * eu
    edu = ea * (dh.abs() + edh) + a.abs() * edh
    mu = u.abs() + eu
    edg = eda * mu * (dh.abs() + edh) + da.abs() * (eu * (dh.abs() + edh) + u.abs() * edh)
    r = max(half, 4 * U)
    eh, edu, edg = (e + r * (v.abs() + e) for e, v in ((eh, h), (edu, du), (edg, dg)))
    acc = lambda k: (k + 8) * U   # noqa: E731
    dx = dg @ Wg.t() + du @ Wu.t()
    ex = edg @ Wg.abs().t() + edu @ Wu.abs().t()
    ex = ex + acc(2 * H) * ((dg.abs() + edg) @ Wg.abs().t() + (du.abs() + edu) @ Wu.abs().t())
    out = dict(dx=(dx, ex + half * (dx.abs() + ex)))
    for n, m, em, v, ev in (("W_gate", x, 0 * x, dg, edg), ("W_up", x, 0 * x, du, edu), ("W_down", h, eh, dF, 0 * dF)):
        d = m.t() @ v
        e = em.t() @ v.abs() + (m.abs() + em).t() @ ev + acc(T + 8) * ((m.abs() + em).t() @ (v.abs() + ev))
        out[n] = (d, e + half * (d.abs() + e))
    return out


def norm_forward(x, gain, eps, half):
    x, w = x.to(F64), gain.to(F64)
    r = 1 / torch.sqrt(x.pow(2).mean(1, keepdim=True) + eps)
    y = x * r * w
    rel = (x.shape[1] + 8) * U            # of r: half the relative error of the mean, a root and a division
    return y, (rel + 4 * U) * y.abs() + half * (1 + rel) * y.abs(), r, rel


def norm_backward(x, gain, dy, eps, half):
    x, w, dy = x.to(F64), gain.to(F64), dy.to(F64)
    _, _, r, rel = norm_forward(x, gain, eps, half)
    v = dy * w
    m = (v * x).mean(1, keepdim=True)
    em = rel * (v * x).abs().mean(1, keepdim=True)
    dx = r * v - x * r ** 3 * m
    ex = (rel + 6 * U) * r * v.abs() + x.abs() * r ** 3 * (em + (3 * rel + 8 * U) * m.abs())
    dw = (dy * x * r).sum(0)
    ew = (rel + (x.shape[0] + 8) * U) * (dy * x * r).abs().sum(0)
    return (dx, ex + half * (dx.abs() + ex)), (dw, ew)


def assert_within(got, ref, what):
    value, bound = ref
    off = (got.detach().cpu().to(F64).reshape(value.shape) - value).abs()
    bad = ~(off <= bound * (1 + 1e-6) + 1e-37)
    if bool(bad.any()):
        i = int((off / (bound + 1e-300)).argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values off; the worst {float(off.reshape(-1)[i]):.3g} "
                             f"where {float(bound.reshape(-1)[i]):.3g} is allowed")


def ffn_inputs(T, C, H, dtype, seed, device="cuda"):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std)   # noqa: E731
    x, dF = n(T, C).to(dtype), n(T, C).to(dtype)
    w = {"W_gate": n(C, H, std=C ** -0.5), "W_up": n(C, H, std=C ** -0.5), "W_down": n(H, C, std=H ** -0.5)}
    return x, dF, w
