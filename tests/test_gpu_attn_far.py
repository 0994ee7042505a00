"""Attention whose scores are far from 0, up to 2^60: finite inputs give finite
answers, and a row whose largest score is far above its others gives that key's
value, weighted with 1, forward and backward.

Keys hold two digits in two channels, so that a row's scores differ by 2^-14 of
them or more and are sums of two products that fp32 holds: the largest is known
without rounding, and all other probabilities are 0 in fp32 from 2^24 on.  What is
left is rounding: the output is the value, rounded once; dv is a sum of rows of dout
in fp32, rounded once; dS is what D-term products of dout with the value and with
the output differ by, so (2 D + 16) 2^-24 of the sum of their absolute products, and
dq and dk are that times a key or a query (and dS rounded, with a bf16 state)."""

import pytest
import torch

from paper_2607_14530_amd import xhc as X
from tests import attn_util as U

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
NAME = {BF: "bf16", F32: "f32"}


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def digits(n, g):
    """n different pairs of digits 1 .. 127, 0 .. 127, in no order."""
    pick = torch.randperm(127 * 128, generator=g)[:n]
    return (1 + pick // 128).float(), (pick % 128).float()


def far_inputs(T, Hq, Hkv, D, dtype, e, seed, scale):
    """Scores of 2^e, of either sign; values and dout as usual."""
    g = torch.Generator().manual_seed(seed)
    x, dout = U.inputs(T, Hq, Hkv, D, F32, seed)
    x[:, :Hq + Hkv] = 0
    size = 2.0 ** (e - 14) / scale               # of a score's smallest difference
    a = 2.0 ** round((e - 14) / 2)
    sign = torch.where(torch.rand(T, Hq, generator=g) < 0.5, -1.0, 1.0)
    x[:, :Hq, 1] = sign * a
    x[:, :Hq, D // 2] = sign * a * 128
    for h in range(Hkv):
        hi, lo = digits(T, g)
        x[:, Hq + h, 1], x[:, Hq + h, D // 2] = lo * (size / a), hi * (size / a)
    return x.to(dtype), dout.to(dtype)


def check(T, S, Hq, Hkv, D, dtype, e, slopes=None, scale=1.0, starts=None, groups=None, seed=0):
    d = X.make_dims(T, 1, 1, 1, 32, S=S, state=NAME[dtype])
    qkv, dout = far_inputs(T, Hq, Hkv, D, dtype, e, seed + e + D, scale)
    sl = None if slopes is None else torch.tensor(slopes, dtype=F32, device="cuda")
    att = X.TrainableAttention(d, X.make_heads(Hq, Hkv, D, scale=scale), slopes=sl)
    span = None if starts is None else att.spans(i32(starts))
    out = att.forward(qkv.cuda(), span)
    dqkv = att.backward(dout.cuda())
    assert bool(torch.isfinite(out.float()).all()) and bool(torch.isfinite(dqkv.float()).all())
    lo, hi = U.spans(T, S, 0, starts)
    j = torch.arange(T)
    seen = (j[None] >= lo[:, None]) & (j[None] < hi[:, None])
    half, g = U.HALF[dtype], Hq // Hkv
    x, go = qkv.to(U.F64), dout.to(U.F64)
    for kh in range(Hkv) if groups is None else groups:
        k, v = x[:, Hq + kh], x[:, Hq + Hkv + kh]
        dk, dv = (torch.zeros(T, D, dtype=U.F64) for _ in range(2))
        edk, edv = torch.zeros_like(dk), torch.zeros_like(dv)
        for h in range(kh * g, kh * g + g):
            s = (x[:, h] @ k.t()).masked_fill(~seen, float("-inf"))
            some = seen.any(1)
            at = s.argmax(1)
            w = some.to(U.F64)[:, None]
            U.assert_within(out[:, h], (w * v[at], half * (w * v[at]).abs()), "out")
            eS = (1 + half) * (2 * D + 16) * U.U * (go[:, h].abs() * v[at].abs()).sum(1, keepdim=True) * w
            U.assert_within(dqkv[:, h], (0 * v, scale * 2 * eS * k[at].abs()), "dq")
            dv.index_add_(0, at, w * go[:, h])
            edv.index_add_(0, at, w * go[:, h].abs())
            edk.index_add_(0, at, scale * 2 * eS * x[:, h].abs())
        U.assert_within(dqkv[:, Hq + kh], (dk, edk), "dk")
        U.assert_within(dqkv[:, Hq + Hkv + kh], (dv, (T * g + 8) * U.U * edv + half * (dv.abs() + edv * (T * g) * U.U)), "dv")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [32, 64, 96, 128])
@pytest.mark.parametrize("e", [24, 27, 30, 33, 60])
def test_few_rows(e, D, dtype):
    check(200, 100, 2, 1, D, dtype, e)
    check(150, 150, 2, 2, D, dtype, e, starts=[0, 70, 130])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [32, 64, 96, 128])
@pytest.mark.parametrize("e", [27, 33, 60])
def test_many_rows(e, D, dtype):
    check(1100, 550, 30, 6, D, dtype, e, groups=[0, 4])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,T,Hq,Hkv", [(64, 200, 2, 1), (128, 200, 2, 1), (64, 1100, 30, 6)])
def test_with_a_bias(D, T, Hq, Hkv, dtype):
    """Far below the scores' differences (2^-14 of 2^40)."""
    check(T, T, Hq, Hkv, D, dtype, 40, slopes=[0.25 / (1 + h) for h in range(Hq)], groups=[0])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale", [2.0 ** 40, 2.0 ** -40])
def test_the_largest_and_smallest_scale(scale, dtype):
    check(150, 150, 2, 1, 64, dtype, 44, scale=scale)
    d = X.make_dims(90, 1, 1, 1, 32, S=90, state=NAME[dtype])      # and ordinary inputs
    qkv, dout = (z.cuda() for z in U.inputs(90, 2, 1, 64, dtype, 3))
    att = X.TrainableAttention(d, X.make_heads(2, 1, 64, scale=scale))
    out, grad = att.forward(qkv).clone(), att.backward(dout).clone()
    assert bool(torch.isfinite(out.float()).all()) and bool(torch.isfinite(grad.float()).all())
    if scale < 1:                                # all scores alike: the mean of what is seen
        v = qkv[:, 3].double()
        mean = v.cumsum(0) / torch.arange(1, 91, device="cuda")[:, None]
        bound = (3 * U.HALF[dtype] + 128 * U.U) * v.abs().cumsum(0) / torch.arange(1, 91, device="cuda")[:, None]
        assert bool(((out.double() - mean[:, None]).abs() <= bound[:, None]).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("new", [1, 5, 40])
@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("e", [24, 33, 60])
def test_over_the_cache(e, D, new, dtype):
    """A digit for each of 110 keys, which the cache holds to 2^-9 of it."""
    B, per, page, Hq, Hkv, n = 2, 4, 32, 6, 2, 110
    g = torch.Generator().manual_seed(e)
    h = X.make_heads(Hq, Hkv, D, rotary=0, scale=1.0)
    x = torch.randn(B * n, Hq + 2 * Hkv, D, generator=g)
    a = 2.0 ** round((e - 7) / 2)
    x[:, Hq:Hq + Hkv] = 0
    for b in range(B):
        for k in range(Hkv):
            x[b * n:(b + 1) * n, Hq + k, 5] = (1 + torch.randperm(n, generator=g)).float() * 2.0 ** (e - 7) / a
    make = lambda T, **kw: X.KVCache(X.make_dims(T, 1, 1, 1, 32, S=1, state=NAME[dtype]), h, None, B, per, page=page,   # noqa: E731
                                     npages=B * per, **kw)
    c = make(B * n)
    pages = torch.randperm(B * per, generator=g).int().view(B, per).cuda()
    args = (i32([0, n, 2 * n]), i32([n, n]), pages)
    c.append(x.to(dtype).cuda(), *args)
    hk, hv = U.held(x.to(dtype)[:, Hq:Hq + Hkv].float()), U.held(x.to(dtype)[:, Hq + Hkv:].float())
    q = torch.zeros(B * new, Hq, D)
    sign = torch.where(torch.rand(B * new, Hq, generator=g) < 0.5, -1.0, 1.0)
    q[:, :, 5] = sign * a
    one = make(B * new, pool=c.pool)
    out = one.attend(q.to(dtype).cuda(), i32([0, new, 2 * new]), i32([n, n]), pages)
    ref = torch.zeros(B * new, Hq, D, dtype=U.F64)
    for t in range(B * new):
        b, p = t // new, n - new + t % new
        rows = slice(b * n, b * n + p + 1)
        for i in range(Hq):
            s = hk[rows, i // 3] @ q[t, i].to(U.F64)
            ref[t, i] = hv[rows, i // 3][s.argmax()]
    U.assert_within(out, (ref, U.HALF[dtype] * ref.abs()), "out")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,Hq,Hkv,D", [(100, 2, 1, 64), (1100, 30, 6, 128)])
def test_a_far_row_leaves_its_neighbours(T, Hq, Hkv, D, dtype):
    """One query whose scores are far: the other rows keep their bits, and so do the gradients of keys behind it."""
    d = X.make_dims(T, 1, 1, 1, 32, S=T, state=NAME[dtype])
    att = X.TrainableAttention(d, X.make_heads(Hq, Hkv, D))
    qkv, dout = (z.cuda() for z in U.inputs(T, Hq, Hkv, D, dtype, 8))
    out, grad = att.forward(qkv).clone(), att.backward(dout).clone()
    t = T // 2
    q2 = qkv.clone()
    q2[t, :Hq] *= 2.0 ** 40
    out2, grad2 = att.forward(q2), att.backward(dout)
    same = torch.ones(T, dtype=torch.bool, device="cuda")
    same[t] = False
    assert torch.equal(out2[same], out[same]) and torch.equal(grad2[same, :Hq], grad[same, :Hq])
    assert torch.equal(grad2[t + 1:], grad[t + 1:])
    assert bool(torch.isfinite(out2.float()).all()) and bool(torch.isfinite(grad2.float()).all())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_far_row_over_the_cache_leaves_its_neighbours(dtype):
    B, per, page, Hq, Hkv, D = 1, 4, 64, 8, 1, 64
    h = X.make_heads(Hq, Hkv, D, rotary=0)
    c = X.KVCache(X.make_dims(200, 1, 1, 1, 32, S=1, state=NAME[dtype]), h, None, B, per, page=page)
    x = U.inputs(200, Hq, Hkv, D, dtype, 9)[0].cuda()
    pages = i32([[3, 1, 0, 2]])
    c.append(x, i32([0, 200]), i32([200]), pages)
    one = X.KVCache(X.make_dims(1, 1, 1, 1, 32, S=1, state=NAME[dtype]), h, None, B, per, page=page, pool=c.pool)
    q = U.inputs(1, Hq, Hkv, D, dtype, 10)[0][:, :Hq].contiguous().cuda()
    args = (i32([0, 1]), i32([200]), pages)
    out = one.attend(q, *args).clone()
    q[0, 5] *= 2.0 ** 40
    out2 = one.attend(q, *args)
    same = [0, 1, 2, 3, 4, 6, 7]
    assert torch.equal(out2[:, same], out[:, same]) and bool(torch.isfinite(out2.float()).all())
