"""The block's activations value by value on the GPU: weights that hand single
columns through, so that F is act(g), the input's gradient act'(g) and act(g),
with no sum to hide an error of the lower tail in."""

import math

import pytest
import torch

from paper_2607_14530_amd import xhc as X

pytestmark = pytest.mark.gpu
F64 = torch.float64
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def expected(g, act, state):
    """act, act' and bounds, of 64-bit g.  Relative errors of the fp32 parts:
    an exponential of x, its argument rounded twice, 2 |x| + 2 units; a
    reciprocal, sum or product one or two; the distribution function of an
    fp32 state 16 (erfc's) and that of its argument (two roundings, 2 g^2 + 2),
    of a bf16 state 2^-21 of 1.  A bf16 state rounds h or dg, once."""
    half = 2.0 ** -8 if state == "bf16" else 0.0
    if act == "silu":
        e = torch.sigmoid(g)
        ee = (2 * g.abs() + 6) * U * e
        a, d = g * e, e * (1 + g * (1 - e))
        # 1 - e: off by e's error and a rounding
        ed = ee * (1 + g.abs()) + a.abs() * (ee + 2 * U) + 2 * U * (e + d.abs())
    else:
        e = 0.5 * torch.erfc(-g / math.sqrt(2.0))
        x = g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
        ee = (2 * g * g + 18) * U * e if state == "f32" else torch.full_like(g, 2.0 ** -21)
        a, d = g * e, e + x
        ed = ee + (g * g + 8) * U * x.abs() + U * d.abs()
    ea = g.abs() * ee + 3 * U * a.abs()
    return (a, ea + half * (a.abs() + ea)), (d, ed + half * (d.abs() + ed))


@pytest.mark.parametrize("T", [1, 64, 300])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("state", ["bf16", "f32"])
def test_activation_and_its_derivative(state, act, T):
    C, H = 32, 16
    g = torch.linspace(-9, 9, T * H).reshape(T, H) if T > 1 else torch.linspace(-7.5, 7.5, H).reshape(1, H)
    x = torch.cat([g, torch.ones(T, H)], 1).to(DT[state])
    eye = torch.eye(H)
    w = {"W_gate": torch.cat([eye, 0 * eye]), "W_up": torch.cat([0 * eye, eye]), "W_down": torch.cat([eye, 0 * eye], 1)}
    ff = X.TrainableFeedForward(X.make_dims(T, 1, 1, 1, C, state=state), H, {k: v.cuda() for k, v in w.items()}, act=act)
    F = ff.forward(x.cuda()).cpu().to(F64)
    dx = ff.backward(torch.cat([torch.ones(T, H), torch.zeros(T, H)], 1).to(DT[state]).cuda()).cpu().to(F64)
    (a, ea), (d, ed) = expected(x[:, :H].to(F64), act, state)
    assert not bool(F[:, H:].any())
    for got, v, tol, what in ((F[:, :H], a, ea, "F"), (dx[:, :H], d, ed, "act'"), (dx[:, H:], a, ea, "du")):
        off = (got - v).abs() - tol * (1 + 1e-9) - 1e-40
        assert bool((off <= 0).all()), (what, float(x[:, :H].reshape(-1)[off.argmax()]), float(off.max()))
