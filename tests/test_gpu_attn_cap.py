"""Attention under a cap where scores come near it, and at the caps' limits.

The cap's derivative is 1 - tanh^2 = 4 e / (1 + e)^2, e = exp(-2 |z|), z = scale q k
/ cap: next to the cap it is as small as e, and a gradient is as exact relative to
it as elsewhere.  So the reference takes z's error, dz, for what it does to that
value: a factor of exp(2 dz) at most.  z carries its product's (D + 8) 2^-24 of the
sum of absolute products; an exponent of 2 |z| log2 e that is formed in four roundings
carries 4 2^-24 of its size, which is 8 |z| 2^-24 of the value; exp2, the reciprocal
or division and the products of the formula some 2^-24 each, 16 in all.  What is below
2^-120 may be cleared."""

import math

import pytest
import torch

from paper_2607_14530_amd import xhc as X
from tests import attn_util as U

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
NAME = {BF: "bf16", F32: "f32"}
TINY = 2.0 ** -120


def scores(q, k, scale, cap, slope, dist):
    """attn_util's scores with the derivative's bound relative to it."""
    D = q.shape[1]
    z = q @ k.t() * scale / cap
    dz = (D + 8) * U.U * (q.abs() @ k.abs().t()) * scale / cap
    s = cap * torch.tanh(z) - slope * dist
    es = dz * cap + 16 * U.U * cap + 4 * U.U * cap * z.abs() + 8 * U.U * (s.abs() + slope * dist)
    e = torch.exp(-2 * z.abs())
    der = 4 * e / (1 + e) ** 2
    eder = der * (torch.exp(2 * dz + (8 * z.abs() + 16) * U.U) - 1) + TINY
    return s, es, der, eder


def run(qkv, dout, Hq, Hkv, cap, dtype, monkeypatch, scale=None, slopes=None):
    T, D = qkv.shape[0], qkv.shape[2]
    monkeypatch.setattr(U, "scores", scores)
    d = X.make_dims(T, 1, 1, 1, 32, S=T, state=NAME[dtype])
    h = X.make_heads(Hq, Hkv, D, cap=cap, scale=scale)
    sl = None if slopes is None else torch.tensor(slopes, dtype=F32, device="cuda")
    att = X.TrainableAttention(d, h, slopes=sl)
    out = att.forward(qkv.cuda())
    dqkv = att.backward(dout.cuda())
    lo, hi = U.spans(T, T)
    ref, dref = U.all_heads(qkv, lo, hi, Hq, Hkv, h.scale, cap, slopes, dout)
    U.assert_within(out, ref, "out")
    for n, a, b in (("dq", 0, Hq), ("dk", Hq, Hq + Hkv), ("dv", Hq + Hkv, Hq + 2 * Hkv)):
        U.assert_within(dqkv[:, a:b], (dref[0][:, a:b], dref[1][:, a:b]), n)


def near(z, T, Hq, Hkv, D, cap, dtype, seed):
    """Queries and keys whose scores lie some 5 % around z caps, those of the second query head around -z."""
    g = torch.Generator().manual_seed(seed)
    x, dout = U.inputs(T, Hq, Hkv, D, F32, seed)
    u = torch.sign(torch.randn(D, generator=g))
    x[:, Hq:Hq + Hkv] = u + 0.2 * x[:, Hq:Hq + Hkv]
    sign = torch.tensor([-1.0 if i % 2 else 1.0 for i in range(Hq)])[None, :, None]
    x[:, :Hq] = sign * z * cap * D ** -0.5 * (u + 0.2 * x[:, :Hq])        # (scale D^-1/2: of D products)
    return x.to(dtype), dout.to(dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("z", [0.5, 4.0, 7.0, 8.5, 12.0, 25.0])
@pytest.mark.parametrize("T,D,cap,slopes", [(70, 64, 20.0, None), (40, 128, 3.0, [0.2, 0.01])])
def test_gradients_where_scores_are_near_the_cap(T, D, cap, slopes, z, dtype, monkeypatch):
    qkv, dout = near(z, T, 2, 1, D, cap, dtype, int(10 * z))
    run(qkv, dout, 2, 1, cap, dtype, monkeypatch, slopes=slopes)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("cap,size", [(2.0 ** -20, 2.0 ** -20), (4096.0, 4096.0), (4096.0, 1.0), (2.0 ** -20, 1.0)])
def test_the_largest_and_smallest_cap(cap, size, dtype, monkeypatch):
    """Scores of about the cap's size, and of about 1: far below the largest cap, and all at the smallest."""
    qkv, dout = U.inputs(100, 4, 2, 64, F32, 31)
    qkv[:, :4] *= size
    run(qkv.to(dtype), dout.to(dtype), 4, 2, cap, dtype, monkeypatch)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scores_that_are_not_bounded_by_fp32(dtype, monkeypatch):
    """Products that overflow: their scores are the cap or less it, and their derivative is 0."""
    T, D = 33, 32
    qkv, dout = U.inputs(T, 1, 1, D, F32, 32)
    qkv[:, :2] = torch.sign(qkv[:, :2]) * 2.0 ** 100
    qkv[:, :2, 1:] = 0
    qkv = qkv.to(dtype)
    d = X.make_dims(T, 1, 1, 1, 32, S=T, state=NAME[dtype])
    att = X.TrainableAttention(d, X.make_heads(1, 1, D, cap=5.0))
    out = att.forward(qkv.cuda()).cpu().double()
    dqkv = att.backward(dout.to(dtype).cuda())
    assert bool((dqkv[:, :2] == 0).all()) and bool(torch.isfinite(dqkv.float()).all())
    s = 5.0 * torch.sign(qkv[:, 0, :1].double() @ qkv[:, 1, :1].double().t())
    p = torch.softmax(s.masked_fill(torch.ones(T, T).triu(1) > 0, -math.inf), 1)
    ref = p @ qkv[:, 2].double()
    # weights and the result rounded, the weights' sum as well, and the reference's 64 bits of 5 as fp32 has them
    bound = (3 * U.HALF[dtype] + 64 * U.U) * (p @ qkv[:, 2].double().abs())
    assert bool(((out[:, 0] - ref).abs() <= bound).all())
