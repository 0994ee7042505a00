"""Rotation, attention and the cache as a program uses them: streams, captured
calls, two calls at once, bad values where nobody looks, offsets past 32 bits,
differences, refused calls of the bundles."""

import pytest
import torch

from paper_2607_14530_amd import xhc as X
from tests import attn_util as U

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
NAME = {BF: "bf16", F32: "f32"}


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def bundle(T, S, Hq, Hkv, D, dtype=BF, train=True, slopes=None, **kw):
    d = X.make_dims(T, 1, 1, 1, 32, S=S, state=NAME[dtype])
    h = X.make_heads(Hq, Hkv, D, **kw)
    return (X.TrainableAttention if train else X.Attention)(d, h, slopes=slopes)


def inputs(T, Hq, Hkv, D, dtype=BF, seed=0):
    qkv, dout = U.inputs(T, Hq, Hkv, D, dtype, seed)
    return qkv.cuda(), dout.cuda()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_seen_does_not_matter(bad, dtype):
    """NaN and infinities in a later token, in another document and in padding: everything that does not see them keeps
    its bits, forward and backward, at every place in a tile."""
    T, Hq, Hkv, D = 200, 4, 2, 64
    starts, prefix = i32([0, 90, 180]), i32([0, 20])
    qkv, dout = inputs(T, Hq, Hkv, D, dtype, 1)
    dout[180:] = 0
    att = bundle(T, T, Hq, Hkv, D, dtype)
    span = att.spans(starts, prefix)
    out, grad = att.forward(qkv, span).clone(), att.backward(dout).clone()
    for t in (60, 89, 150, 190):
        q2, d2 = qkv.clone(), dout.clone()
        q2[t] = bad
        d2[t] = bad
        out2 = att.forward(q2, span).clone()
        grad2 = att.backward(d2).clone()
        if t >= 180:                             # padding: nobody sees it, it sees nobody
            same = torch.ones(T, dtype=torch.bool)
            same[t] = False
            gsame = same
        else:
            end = 90 if t < 90 else 180
            same = torch.ones(T, dtype=torch.bool)
            same[t:end] = False                  # who sees it
            gsame = torch.ones(T, dtype=torch.bool)
            gsame[0 if t < 90 else 90:end] = False
            assert bool((~torch.isfinite(out2[t:end].float())).any(-1).all())
        assert torch.equal(out2[same.cuda()], out[same.cuda()]), t
        assert torch.equal(grad2[gsame.cuda()], grad[gsame.cuda()]), t
    assert bool((out[180:] == 0).all()) and bool((grad[180:] == 0).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("cap", [0.0, 30.0])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_one_bad_channel_of_a_query_or_its_gradient(bad, cap, dtype):
    """A query, or a row of dout, with one channel that is not finite only changes its own row and the gradients of keys
    that it sees (a cap bounds the scores of an infinite query, whose sums are then finite)."""
    T, Hq, Hkv, D = 330, 6, 2, 64
    starts = i32([0, 100, 300])
    qkv, dout = inputs(T, Hq, Hkv, D, dtype, 2)
    att = bundle(T, T, Hq, Hkv, D, dtype, cap=cap)
    span = att.spans(starts)
    out, grad = att.forward(qkv, span).clone(), att.backward(dout).clone()
    for t in (0, 63, 99, 130, 255, 299):
        first, end = (0, 100) if t < 100 else (100, 300)
        for of_query in (True, False):
            q2, d2 = qkv.clone(), dout.clone()
            (q2 if of_query else d2)[t, 4, 37] = bad             # query head 4: of key and value head 1
            out2, grad2 = att.forward(q2, span).clone(), att.backward(d2).clone()
            same = torch.ones(T, Hq, dtype=torch.bool, device="cuda")
            same[t, 4] = not of_query
            assert torch.equal(out2[same], out[same]), (t, of_query)
            same = torch.ones(T, Hq + 2 * Hkv, dtype=torch.bool, device="cuda")
            same[t, 4] = False
            same[first:t + 1, Hq + 1] = same[first:t + 1, Hq + Hkv + 1] = False
            assert torch.equal(grad2[same], grad[same]), (t, of_query)
            row = grad2[t, 4].float()
            if of_query and cap and bad == bad:  # scores of an infinite query are cap or -cap, where tanh' = 0
                assert bool((row == 0).all()), t
                k, v = (qkv[first:t + 1, h].double() for h in (Hq + 1, Hq + Hkv + 1))
                p = torch.softmax(cap * torch.sign(bad * k[:, 37]), 0)
                # the row's own values are among those; p is rounded, and so is what it is divided by, and the result
                bound = 3 * torch.finfo(dtype).eps / 2 if dtype is BF else 2.0 ** -16
                err = (out2[t, 4].double() - (p[:, None] * v).sum(0)).abs().max()
                assert float(err) <= bound * float(v.abs().max()), (t, float(err))
            else:
                assert not bool(torch.isfinite(row).all()), (t, of_query)
            assert bool(torch.isfinite(grad2[t + 1:end].float()).all()), (t, of_query)


def test_the_same_twice():
    """The same bits from call to call, whatever the buffers held."""
    T, Hq, Hkv, D = 700, 8, 2, 128
    qkv, dout = inputs(T, Hq, Hkv, D)
    att = bundle(T, 350, Hq, Hkv, D, cap=10.0)
    a, b = att.forward(qkv).clone(), att.backward(dout).clone()
    for fill in (0, 255):
        for t in (att.ws, att.saved):
            t.fill_(fill)
        att.out.fill_(float("nan"))
        att.dqkv.fill_(float("nan"))
        assert torch.equal(att.forward(qkv), a)
        assert torch.equal(att.backward(dout), b)


def test_workspace_is_not_written_past_its_end():
    for T, Hq, Hkv, D, dtype in ((65, 4, 1, 64, BF), (130, 2, 2, 96, F32), (300, 8, 2, 128, BF)):
        qkv, dout = inputs(T, Hq, Hkv, D, dtype)
        att = bundle(T, T, Hq, Hkv, D, dtype)
        for name in ("ws", "saved"):
            t = getattr(att, name)
            big = torch.full((t.numel() + 4096,), 77, dtype=torch.uint8, device="cuda")
            setattr(att, name, big[:t.numel()])
            setattr(att, name + "_all", big)
        att.forward(qkv)
        att.backward(dout)
        for name in ("ws", "saved"):
            t, big = getattr(att, name), getattr(att, name + "_all")
            assert bool((big[t.numel():] == 77).all()), name


def test_other_stream_and_two_at_once():
    T, Hq, Hkv, D = 900, 8, 4, 64
    qkv, dout = inputs(T, Hq, Hkv, D)
    ref = bundle(T, 450, Hq, Hkv, D)
    out, grad = ref.forward(qkv).clone(), ref.backward(dout).clone()
    streams = [torch.cuda.Stream() for _ in range(2)]
    atts = [bundle(T, 450, Hq, Hkv, D) for _ in range(2)]
    rots = []
    torch.cuda.synchronize()
    for _ in range(5):
        for s, att in zip(streams, atts):
            att.forward(qkv, stream=s)
            att.backward(dout, stream=s)
    torch.cuda.synchronize()
    for att in atts:
        assert torch.equal(att.out, out) and torch.equal(att.dqkv, grad)
    table = X.rotation_table(450, D)
    rot = X.Rotation(ref.d, ref.h, table)
    want = rot.forward(qkv).clone()
    with torch.cuda.stream(streams[0]):
        rots.append(X.Rotation(ref.d, ref.h, table).forward(qkv))
    streams[0].synchronize()
    assert torch.equal(rots[0], want)


def test_captured_training_step():
    """A captured forward and backward, replayed on new values with eager work between, next to an eager one of its own
    buffers."""
    T, Hq, Hkv, D = 390, 6, 2, 128
    qkv, dout = inputs(T, Hq, Hkv, D)
    starts = i32([0, 100, 260, 380])
    att, eager = bundle(T, T, Hq, Hkv, D), bundle(T, T, Hq, Hkv, D)
    table = X.rotation_table(T, D)
    rot = X.Rotation(att.d, att.h, table)

    def step(a, r):
        x = r.forward(qkv)
        o = a.forward(x, a.spans(starts))
        return o, r.backward(a.backward(dout))

    step(att, rot)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, grad = step(att, rot)
    rot2 = X.Rotation(att.d, att.h, table)
    for seed in range(4):
        q, d = inputs(T, Hq, Hkv, D, seed=seed)
        qkv.copy_(q)
        dout.copy_(d)
        starts.copy_(i32([0, 50 + 30 * seed, 260, 380 - seed]))
        g.replay()
        torch.cuda.synchronize()
        o2, g2 = step(eager, rot2)
        assert torch.equal(out, o2) and torch.equal(grad, g2)


def test_captured_decoding():
    """Captured appends and attention follow the lengths and page table on the device."""
    B, page, per, Hq, Hkv, D = 5, 32, 8, 8, 2, 64
    h = X.make_heads(Hq, Hkv, D)
    table = X.rotation_table(page * per, D)
    one, many = (X.make_dims(T, 1, 1, 1, 32, S=1) for T in (B, 5 * 100))
    pages = torch.randperm(B * per, device="cuda").int().view(B, per)
    starts1 = i32(list(range(B + 1)))
    caches = []
    for _ in range(2):
        c = X.KVCache(many, h, table, B, per, page=page)
        g = torch.Generator(device="cuda").manual_seed(3)
        qkv = torch.randn(500, Hq + 2 * Hkv, D, device="cuda", generator=g).bfloat16()
        c.append(qkv, i32([0, 10, 30, 200, 201, 500]), i32([10, 20, 170, 1, 256 - 57 + 100 - 0]).clamp(max=256), pages)
        caches.append(X.KVCache(one, h, table, B, per, page=page, pool=c.pool))
    lens = i32([10, 20, 170, 1, 200])
    x = torch.randn(B, Hq + 2 * Hkv, D, device="cuda").bfloat16()

    def step(c):
        q = c.append(x, starts1, lens, pages)
        return c.attend(q, starts1, lens, pages)

    lens += 1
    step(caches[0])
    step(caches[1])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step(caches[0])
    for k in range(6):
        x.copy_(torch.randn(B, Hq + 2 * Hkv, D, device="cuda"))
        lens += 1
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, step(caches[1])), k
        assert torch.equal(caches[0].pool, caches[1].pool)


def test_two_pools_of_heads_do_not_meet():
    """What is not of the call's blocks keeps its bytes: other pages, and of the pages written other heads' blocks and
    tokens that were there."""
    B, page, per, Hq, Hkv, D = 2, 64, 2, 4, 2, 128
    h = X.make_heads(Hq, Hkv, D)
    d = X.make_dims(3, 1, 1, 1, 32, S=1)
    c = X.KVCache(d, h, X.rotation_table(page * per, D), B, per, page=page, npages=6)
    c.pool.random_(0, 256)
    before = c.pool.clone()
    pages = i32([[4, 1], [2, 5]])
    qkv = torch.randn(3, Hq + 2 * Hkv, D, device="cuda").bfloat16()
    c.append(qkv, i32([0, 1, 3]), i32([66, 34]), pages)      # token 65 of page 1, tokens 32 and 33 of page 2
    changed = (c.pool != before).view(6, Hkv, 2, -1).any(-1).cpu()
    want = torch.zeros(6, Hkv, 2, dtype=torch.bool)
    want[1, :, 0] = True
    want[2, :, 1] = True
    assert torch.equal(changed, want)
    n = (c.pool != before).view(6, Hkv, 2, -1).sum(-1).cpu()
    # a token has D / 2 + D / 16 bytes of keys and as many of values, whose nibbles share bytes with a neighbour's
    assert int(n[1].max()) <= D // 2 + D // 16 + D + D // 16
    assert int(n[2].max()) <= 2 * (D // 2 + D // 16) + D + 2 * (D // 16)


def test_offsets_past_32_bits():
    """A pool past 4 GiB, whose last pages are in use, and token rows past 2^32 bytes."""
    page, D, Hq, Hkv = 1024, 128, 8, 8
    npages = (5 << 30) // (Hkv * page * 144)
    h = X.make_heads(Hq, Hkv, D)
    table = X.rotation_table(2 * page, D)
    d = X.make_dims(1500, 1, 1, 1, 32, S=1)
    x = torch.randn(1500, Hq + 2 * Hkv, D, device="cuda").bfloat16()
    q = torch.randn(1, Hq, D, device="cuda").bfloat16()
    outs = []
    for n, pages in ((npages, i32([[npages - 1, npages - 2]])), (3, i32([[1, 2]]))):
        c = X.KVCache(d, h, table, 1, 2, page=page, npages=n)
        c.append(x, i32([0, 1500]), i32([1500]), pages)
        c1 = X.KVCache(X.make_dims(1, 1, 1, 1, 32, S=1), h, table, 1, 2, page=page, npages=n, pool=c.pool)
        outs.append(c1.attend(q, i32([0, 1]), i32([1500]), pages).clone())
        del c, c1
        torch.cuda.empty_cache()
    assert torch.equal(*outs)
    # rows: only the last sequence of a long batch has values that matter
    T, S, Hq, Hkv, D = 1 << 19, 512, 32, 2, 128
    tail, dt = U.inputs(S, Hq, Hkv, D, BF, 4)
    lo, hi = U.spans(S, S, 100)
    ref, dref = U.all_heads(tail, lo, hi, Hq, Hkv, D ** -0.5, dout=dt)
    qkv = torch.zeros(T, Hq + 2 * Hkv, D, dtype=BF, device="cuda")
    qkv[-S:] = tail.cuda()
    big = bundle(T, S, Hq, Hkv, D, window=100)
    dout = torch.zeros(T, Hq, D, dtype=BF, device="cuda")
    dout[-S:] = dt.cuda()
    assert qkv.numel() * 2 > 1 << 32 and dout.numel() * 2 >= 1 << 32
    U.assert_within(big.forward(qkv)[-S:], ref, "out")
    U.assert_within(big.backward(dout)[-S:], dref, "dqkv")
    table = X.rotation_table(S, D)
    cs = table.cpu()
    y = tail.float()
    y[:, :Hq + Hkv] = U.rotated(tail[:, :Hq + Hkv], cs, D, "halves")
    assert torch.equal(X.Rotation(big.d, big.h, table).forward(qkv)[-S:].cpu(), y.to(BF))


def test_gradients_match_differences():
    """fp32: the loss's change along a direction.  Its derivative is formed from losses 2^-6 apart (relative to inputs of
    about 1), off by a third derivative's share (below 2^-10 of the sizes here) and 2^-24 2^6 of the loss's terms."""
    T, Hq, Hkv, D = 90, 4, 2, 64
    qkv, dout = inputs(T, Hq, Hkv, D, F32, 5)
    att = bundle(T, T, Hq, Hkv, D, F32, cap=4.0, slopes=torch.tensor([0.1, 0.0, 0.3, 0.02], device="cuda"))
    span = att.spans(i32([0, 40, 88]), i32([10, 40]))
    loss = lambda x: float((att.forward(x, span).double() * dout.double()).sum())   # noqa: E731
    v = torch.randn(qkv.shape, generator=torch.Generator().manual_seed(6)).cuda()
    v[:, :, 1:] = 0                              # few channels, so that higher derivatives stay small
    s = 2.0 ** -6
    diff = (loss(qkv + s * v) - loss(qkv - s * v)) / (2 * s)
    att.forward(qkv, span)
    g = att.backward(dout)
    assert abs(diff - float((g.double() * v.double()).sum())) <= 2.0 ** -9 * float((g.double() * v.double()).abs().sum())


def test_refused_calls_of_the_bundles():
    T, Hq, Hkv, D = 16, 4, 2, 64
    qkv, dout = inputs(T, Hq, Hkv, D)
    att = bundle(T, T, Hq, Hkv, D)
    with pytest.raises(ValueError, match="without a forward"):
        att.backward(dout)
    for bad in (qkv[:, :7], qkv.float(), qkv.cpu()):
        with pytest.raises(ValueError):
            att.forward(bad)
    with pytest.raises(ValueError):
        att.forward(qkv, span=torch.zeros(T, 2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        att.forward(qkv.transpose(0, 1).contiguous().transpose(0, 1))        # not contiguous
    att.forward(qkv)
    with pytest.raises(ValueError):
        att.forward(qkv[:8])
    att.backward(dout)                           # of the forward that ran
    with pytest.raises(ValueError):
        att.spans(i32([]))
    with pytest.raises(ValueError):
        att.spans(i32([0, 4, 16]), i32([1]))
    with pytest.raises(ValueError):
        X.TrainableAttention(att.d, att.h, slopes=torch.zeros(3, device="cuda"))
    rot = X.Rotation(att.d, att.h, X.rotation_table(T, D))
    with pytest.raises(ValueError):
        rot.forward(qkv.float())
    with pytest.raises(ValueError):
        rot.forward(qkv, pos=torch.zeros(T, device="cuda"))
    with pytest.raises(ValueError):
        X.Rotation(att.d, att.h, X.rotation_table(T, D // 2))
    with pytest.raises(X.XhcError):
        X.Rotation(att.d, att.h, X.rotation_table(T - 1, D)).forward(qkv)
    with pytest.raises(ValueError):
        X.KVCache(att.d, att.h, X.rotation_table(64, D), 2, 2, page=40)
    c = X.KVCache(att.d, att.h, X.rotation_table(64, D), 2, 2, page=32)
    args = (i32([0, 8, 16]), i32([8, 8]), i32([[0, 1], [2, 3]]))
    c.append(qkv, *args)
    for k in range(3):
        wrong = list(args)
        wrong[k] = wrong[k][:1]
        with pytest.raises(ValueError):
            c.append(qkv, *wrong)
        with pytest.raises(ValueError):
            c.attend(c.q, *wrong)
        with pytest.raises(ValueError):
            c.read(*wrong)
    with pytest.raises(ValueError):
        X.KVCache(att.d, att.h, X.rotation_table(64, D), 2, 2, page=32, pool=c.pool[:-1])
    with pytest.raises(X.XhcError):
        X.KVCache(att.d, att.h, X.rotation_table(63, D), 2, 2, page=32).append(qkv, *args)


def test_empty_batches():
    d = X.make_dims(0, 1, 1, 1, 32, S=1)
    h = X.make_heads(4, 2, 64)
    qkv = torch.empty(0, 8, 64, dtype=BF, device="cuda")
    att = X.TrainableAttention(d, h)
    assert att.forward(qkv).shape == (0, 4, 64)
    assert att.backward(torch.empty(0, 4, 64, dtype=BF, device="cuda")).shape == (0, 8, 64)
    assert X.Rotation(d, h, X.rotation_table(4, 64)).forward(qkv).shape == (0, 8, 64)
    c = X.KVCache(d, h, X.rotation_table(64, 64), 2, 2, page=32)
    args = (i32([0, 0, 0]), i32([3, 0]), i32([[0, 1], [2, 3]]))
    q = c.append(qkv, *args)
    assert q.shape == (0, 4, 64) and c.attend(q, *args).shape == (0, 4, 64) and c.read(*args)[0].shape == (0, 2, 64)
