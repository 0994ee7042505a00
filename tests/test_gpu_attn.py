"""Rotation and attention on the GPU against the formulas in 64 bits, value by
value within bounds that count the roundings."""

import pytest
import torch

from paper_2607_14530_amd import xhc as X
from tests import attn_util as U

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
NAME = {BF: "bf16", F32: "f32"}


def run(T, S, Hq, Hkv, D, dtype, seed=0, window=0, cap=0.0, slopes=None, starts=None, prefix=None, span=None, q_scale=1.0,
        train=True):
    d = X.make_dims(T, 1, 1, 1, 32, S=S, state=NAME[dtype])
    h = X.make_heads(Hq, Hkv, D, window=window, cap=cap)
    qkv, dout = U.inputs(T, Hq, Hkv, D, dtype, seed)
    qkv[:, :Hq] *= q_scale
    sl = None if slopes is None else torch.tensor(slopes, dtype=F32, device="cuda")
    att = (X.TrainableAttention if train else X.Attention)(d, h, slopes=sl)
    if span is not None:
        lo, hi = span
        sp = torch.stack([lo, hi], 1).int().cuda()
        lo, hi = lo.clamp(0, T), hi.clamp(0, T)
    else:
        lo, hi = U.spans(T, S, window, starts, prefix)
        sp = None
        if starts is not None:
            i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")   # noqa: E731
            sp = att.spans(i32(starts), None if prefix is None else i32(prefix))
            some = hi > lo
            got = sp.cpu().long()
            assert bool((got[some, 0] == lo[some]).all() and (got[some, 1] == hi[some]).all())
            assert bool((got[~some, 0] >= got[~some, 1]).all())
    out = att.forward(qkv.cuda(), sp)
    ref, dref = U.all_heads(qkv, lo, hi, Hq, Hkv, D ** -0.5, cap, slopes, dout if train else None)
    U.assert_within(out, ref, "out")
    if train:
        dqkv = att.backward(dout.cuda())
        for n, a, b in (("dq", 0, Hq), ("dk", Hq, Hq + Hkv), ("dv", Hq + Hkv, Hq + 2 * Hkv)):
            U.assert_within(dqkv[:, a:b], (dref[0][:, a:b], dref[1][:, a:b]), n)
    return att


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [32, 64, 96, 128])
@pytest.mark.parametrize("T,S,Hq,Hkv", [(1, 1, 1, 1), (2, 1, 2, 1), (65, 65, 2, 2), (200, 100, 6, 2), (259, 259, 3, 1)])
def test_causal(T, S, Hq, Hkv, D, dtype):
    run(T, S, Hq, Hkv, D, dtype, seed=T + D)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,Hq,Hkv,D,kw", [
    (513, 1, 1, 96, {}), (900, 2, 1, 64, dict(cap=15.0)), (1100, 3, 3, 128, dict(window=300)),
    (777, 4, 2, 32, dict(slopes=[0.5, 0.1, 0.02, 0.0], starts=[0, 3, 600, 770], prefix=[1, 400, 0]))])
def test_few_heads_of_many_tokens(T, Hq, Hkv, D, kw, dtype):
    """Sums of dq, dk and dv in slices of the keys and queries, some of which have none."""
    run(T, T, Hq, Hkv, D, dtype, seed=T, **kw)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("cap,slopes,window", [(2.0, None, 0), (0.0, [0.25, 0.01, 0.5, 1.0], 0), (20.0, [0.1, 0.2, 0.0, 0.4], 70),
                                               (0.0, None, 1), (0.0, None, 64)])
def test_cap_bias_window(cap, slopes, window, dtype):
    run(300, 150, 4, 2, 64, dtype, seed=5, cap=cap, slopes=slopes, window=window, q_scale=3.0)
    run(130, 130, 4, 4, 128, dtype, seed=6, cap=cap, slopes=slopes, window=window)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("starts,prefix,window", [
    ([0, 1, 2, 70, 70, 199, 290], None, 0),              # of one token, an empty one, padding behind the last
    ([3, 64, 128, 300], [5, 64, 0], 0),                  # tokens before the first
    ([0, 150, 300], [150, 1000], 0),                     # nothing but a prefix, one cut at its document's end
    ([0, 100, 300], [40, 90], 30),
    ([0], None, 0),                                      # no document at all: every row empty
])
def test_documents(starts, prefix, window, dtype):
    run(300, 300, 4, 1, 64, dtype, seed=7, starts=starts, prefix=prefix, window=window)
    run(300, 300, 2, 2, 128, dtype, seed=8, starts=starts, prefix=prefix, window=window, cap=5.0, slopes=[0.1, 0.02])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_any_spans(dtype):
    """Spans of no order, some empty, some reaching past the ends."""
    T = 270
    g = torch.Generator().manual_seed(11)
    lo = torch.randint(-50, T + 20, (T,), generator=g)
    hi = lo + torch.randint(-30, 200, (T,), generator=g)
    lo[5], hi[5] = -2 ** 31, 2 ** 31 - 1
    lo[6], hi[6] = 2 ** 31 - 1, -2 ** 31
    run(T, T, 4, 2, 64, dtype, seed=12, span=(lo, hi), slopes=[0.1, 0.0, 0.3, 0.01])
    run(T, T, 3, 1, 96, dtype, seed=13, span=(lo, hi), train=False)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
@pytest.mark.parametrize("T,S,Hq,Hkv,D,R", [(1, 1, 1, 1, 32, 32), (77, 77, 6, 2, 96, 48), (130, 65, 32, 8, 128, 128),
                                            (64, 8, 40, 40, 64, 16), (9, 9, 2, 1, 64, 0)])
def test_rotation(T, S, Hq, Hkv, D, R, pairs, dtype):
    """The formula's bits: fp32 products and sums rounded one by one, then the state dtype's rounding."""
    d = X.make_dims(T, 1, 1, 1, 32, S=S, state=NAME[dtype])
    h = X.make_heads(Hq, Hkv, D, rotary=R, pairing=pairs)
    P = S + 3
    table = X.rotation_table(P, R)
    rot = X.Rotation(d, h, table)
    x, _ = U.inputs(T, Hq, Hkv, D, dtype, T)
    g = torch.Generator().manual_seed(T)
    pos = torch.randint(-2, P + 2, (T,), generator=g, dtype=torch.int32)
    for p in (None, pos):
        at = torch.arange(T) % S if p is None else p.long()
        inside = ((at >= 0) & (at < P))[:, None, None]
        cs = table.cpu()[at.clamp(0, P - 1)]
        for inverse in (False, True):
            y = x.float().clone()
            y[:, :Hq + Hkv] = torch.where(inside, U.rotated(x[:, :Hq + Hkv], cs, R, pairs, inverse), y[:, :Hq + Hkv])
            y = y.to(dtype)
            f = rot.backward if inverse else rot.forward
            dp = None if p is None else p.cuda()
            assert torch.equal(f(x.cuda(), dp).cpu(), y)
            z = x.cuda()
            assert f(z, dp, out=z) is z and torch.equal(z.cpu(), y)
