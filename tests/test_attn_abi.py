"""Rotation, attention and the paged cache refuse what they do not take before
any launch (no GPU needed: nothing below is dereferenced)."""

import ctypes
import re

import pytest
import torch

from paper_2607_14530_amd import xhc as X
from tests import attn_util as U

A = [(i + 1) << 40 for i in range(14)]       # distinct aligned addresses, far apart
BIG = 1 << 50


def dims(**kw):
    base = dict(T=64, N=1, k=1, m=1, C=32, S=64)
    base.update(kw)
    return X.make_dims(**base)


def heads(Hq=4, Hkv=2, D=64, **kw):
    return X.make_heads(Hq, Hkv, D, **kw)


def changed(h, **kw):
    for n, v in kw.items():
        setattr(h, n, v)
    return h


def cache(page=64, npages=8, B=2, per_seq=4):
    return X.Cache(page, npages, B, per_seq)


def with_at(p, i, v):
    return [v if j == i else a for j, a in enumerate(p)]


def rotate(d, h, p, positions=64, inverse=0):         # in, pos, table, out
    return X.lib().xhc_rotate(ctypes.byref(d), ctypes.byref(h), p[0], p[1], p[2], positions, inverse, p[3], None)


def spans(d, h, n, p):                                # starts, prefix, span
    return X.lib().xhc_attn_spans(ctypes.byref(d), ctypes.byref(h), n, *p, None)


def attn(d, h, p):                                    # qkv, span, slopes, out, saved
    return X.lib().xhc_attn(ctypes.byref(d), ctypes.byref(h), *p, None)


def attn_bwd(d, h, p, ws=BIG):                        # qkv, span, slopes, out, saved, dout, dqkv, workspace
    return X.lib().xhc_attn_bwd(ctypes.byref(d), ctypes.byref(h), *p, ws, None)


def append(d, h, c, p, positions=256):                # qkv, table, starts, lens, pages, pool, q
    return X.lib().xhc_cache_append(ctypes.byref(d), ctypes.byref(h), ctypes.byref(c), p[0], p[1], positions, *p[2:], None)


def read(d, h, c, p):                                 # starts, lens, pages, pool, k, v
    return X.lib().xhc_cache_read(ctypes.byref(d), ctypes.byref(h), ctypes.byref(c), *p, None)


def attend(d, h, c, p, ws=BIG):                       # q, slopes, starts, lens, pages, pool, out, workspace
    return X.lib().xhc_attn_cache(ctypes.byref(d), ctypes.byref(h), ctypes.byref(c), *p, ws, None)


CALLS = [(lambda d, h: rotate(d, h, A[:4])), (lambda d, h: spans(d, h, 3, A[:3])), (lambda d, h: attn(d, h, A[:5])),
         (lambda d, h: attn_bwd(d, h, A[:8])), (lambda d, h: append(d, h, cache(), A[:7])),
         (lambda d, h: read(d, h, cache(), A[:6])), (lambda d, h: attend(d, h, cache(), A[:8]))]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("kw,status", [
    (dict(Hkv=0), X.XHC_EINVAL), (dict(Hq=0), X.XHC_EINVAL), (dict(Hq=5), X.XHC_EINVAL), (dict(R=-16), X.XHC_EINVAL),
    (dict(R=80), X.XHC_EINVAL), (dict(D=0, R=0), X.XHC_EINVAL), (dict(pairs=2), X.XHC_EINVAL),
    (dict(window=-1), X.XHC_EINVAL), (dict(scale=0.0), X.XHC_EINVAL), (dict(scale=float("nan")), X.XHC_EINVAL),
    (dict(scale=float("inf")), X.XHC_EINVAL), (dict(cap=-1.0), X.XHC_EINVAL), (dict(cap=float("inf")), X.XHC_EINVAL),
    (dict(D=48, R=48), X.XHC_EUNSUPPORTED), (dict(D=160), X.XHC_EUNSUPPORTED), (dict(R=24), X.XHC_EUNSUPPORTED),
    (dict(cap=4097.0), X.XHC_EUNSUPPORTED), (dict(cap=2.0 ** -21), X.XHC_EUNSUPPORTED),
    (dict(scale=2.0 ** 41), X.XHC_EUNSUPPORTED), (dict(scale=2.0 ** -41), X.XHC_EUNSUPPORTED),
    (dict(Hq=1024), X.XHC_EUNSUPPORTED), (dict(Hq=1024, Hkv=1024), X.XHC_EUNSUPPORTED),
])
def test_heads_refused(call, kw, status):
    assert call(dims(), changed(heads(), **kw)) == status


@pytest.mark.parametrize("call", CALLS)
def test_dims_refused(call):
    assert call(dims(S=5), heads()) == X.XHC_EINVAL
    assert call(dims(T=(1 << 23) + 1, S=1), heads()) == X.XHC_EUNSUPPORTED
    assert call(dims(T=1 << 23, S=1), heads(62, 2)) == X.XHC_EUNSUPPORTED
    assert call(dims(T=0, S=1), heads()) == X.XHC_OK


def refused(call, p, optional, align):
    """Each pointer missing (but the optional ones) and each misaligned."""
    for i in range(len(p)):
        if i not in optional:
            assert call(with_at(p, i, None)) == X.XHC_EINVAL, i
        assert call(with_at(p, i, p[i] + align[i] // 2)) == X.XHC_EUNSUPPORTED, i


def overlaps(call, p, sizes, outs):
    """Each output laid over each other buffer's last bytes, and its own over theirs."""
    for o in outs:
        for i in range(len(p)):
            if i == o:
                continue
            step = 256
            assert call(with_at(p, o, p[i] + (sizes[i] - 1) // step * step)) == X.XHC_EINVAL, (o, i)
            assert call(with_at(p, i, p[o] + (sizes[o] - 1) // step * step)) == X.XHC_EINVAL, (o, i)


QKV, ROWS, KV = 64 * 8 * 64 * 2, 64 * 4 * 64 * 2, 64 * 2 * 64 * 2


def test_rotate_refusals():
    d, h = dims(), heads()
    call = lambda p: rotate(d, h, p)   # noqa: E731
    refused(call, A[:4], {1}, [16, 4, 16, 16])
    overlaps(call, A[:4], [QKV, 256, 64 * 64 * 4, QKV], [3])
    assert rotate(d, h, A[:4], positions=-1) == X.XHC_EINVAL
    assert rotate(d, h, A[:4], inverse=2) == X.XHC_EINVAL
    assert rotate(d, h, with_at(A[:4], 1, None), positions=63) == X.XHC_EINVAL


def test_spans_refusals():
    d, h = dims(), heads()
    assert spans(d, h, -1, A[:3]) == X.XHC_EINVAL
    assert spans(d, h, 1, [None, None, A[2]]) == X.XHC_EINVAL
    assert spans(d, h, 0, [None, A[1], A[2]]) == X.XHC_EINVAL
    assert spans(d, h, 3, [A[0], A[1], None]) == X.XHC_EINVAL
    for i, off in ((0, 2), (1, 2), (2, 4)):
        assert spans(d, h, 3, with_at(A[:3], i, A[i] + off)) == X.XHC_EUNSUPPORTED
    assert spans(d, h, 3, [A[2] + 504, A[1], A[2]]) == X.XHC_EINVAL
    assert spans(d, h, 3, [A[0], A[2] + 8, A[2]]) == X.XHC_EINVAL


def test_attn_refusals():
    d, h = dims(), heads()
    saved = X.xhc_attn_saved_bytes(d, h)
    assert saved == 64 * 4 * 4 + ROWS and X.xhc_attn_saved_bytes(dims(state="f32"), h) == 64 * 4 * 4
    refused(lambda p: attn(d, h, p), A[:5], {1, 2, 4}, [16, 8, 4, 16, 16])
    overlaps(lambda p: attn(d, h, p), A[:5], [QKV, 512, 16, ROWS, saved], [3, 4])
    refused(lambda p: attn_bwd(d, h, p), A[:8], {1, 2}, [16, 8, 4, 16, 16, 16, 16, 16])
    need = X.xhc_attn_workspace_bytes(d, h)
    overlaps(lambda p: attn_bwd(d, h, p), A[:8], [QKV, 512, 16, ROWS, saved, ROWS, QKV, need], [6, 7])
    assert need > 0 and attn_bwd(d, h, A[:8], need - 1) == X.XHC_EWORKSPACE
    assert X.xhc_attn_workspace_bytes(d, heads(D=160)) == 0
    for state in ("bf16", "f32"):                  # no token, one, and few of few heads
        none, one = (X.xhc_attn_workspace_bytes(dims(T=t, state=state), heads(Hq=1, Hkv=1)) for t in (0, 1))
        assert none <= one < 1 << 20


def test_cache_refusals():
    d, h, c = dims(), heads(), cache()
    pool = X.xhc_cache_bytes(h, c)
    # 8 pages of 2 blocks for 2 heads; a block has 32 tokens' keys and values of 64 / 2 + 64 / 16 bytes
    assert pool == 8 * 2 * 2 * 32 * 2 * (32 + 4)
    refused(lambda p: append(d, h, c, p), A[:7], {6}, [16, 16, 4, 4, 4, 256, 16])
    overlaps(lambda p: append(d, h, c, p), A[:7], [QKV, 256 * 64 * 4, 12, 8, 32, pool, ROWS], [5, 6])
    assert append(d, h, c, A[:7], positions=255) == X.XHC_EINVAL
    refused(lambda p: read(d, h, c, p), A[:6], set(), [4, 4, 4, 256, 16, 16])
    overlaps(lambda p: read(d, h, c, p), A[:6], [12, 8, 32, pool, KV, KV], [4, 5])
    refused(lambda p: attend(d, h, c, p), A[:8], {1}, [16, 4, 4, 4, 4, 256, 16, 16])
    need = X.xhc_attn_cache_workspace_bytes(d, h, c)
    overlaps(lambda p: attend(d, h, c, p), A[:8], [ROWS, 16, 12, 8, 32, pool, ROWS, need], [6, 7])
    assert need > 0 and attend(d, h, c, A[:8], need - 1) == X.XHC_EWORKSPACE
    for kw, status in ((dict(page=0), X.XHC_EINVAL), (dict(npages=0), X.XHC_EINVAL), (dict(B=0), X.XHC_EINVAL),
                       (dict(per_seq=0), X.XHC_EINVAL), (dict(page=48), X.XHC_EUNSUPPORTED),
                       (dict(page=1056), X.XHC_EUNSUPPORTED), (dict(B=65537), X.XHC_EUNSUPPORTED),
                       (dict(page=1024, per_seq=16385), X.XHC_EUNSUPPORTED)):
        bad = cache(**kw)
        assert append(d, h, bad, A[:7], positions=1 << 30) == status
        assert read(d, h, bad, A[:6]) == status
        assert attend(d, h, bad, A[:8]) == status
        assert X.xhc_cache_bytes(h, bad) == 0 and X.xhc_attn_cache_workspace_bytes(d, h, bad) == 0


@pytest.mark.parametrize("name,cls", [("xhc_heads", X.Heads), ("xhc_cache", X.Cache)])
def test_struct_fields_match_header(name, cls):
    text = re.sub(r"/\*.*?\*/", "", open(X.HEADER).read(), flags=re.S)
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), text, flags=re.S).group(1)
    assert re.findall(r"\b(\w+)\s*;", body) == [f[0] for f in cls._fields_]


def test_make_heads():
    h = X.make_heads(8, 2, 64)
    assert (h.R, h.pairs, h.window, h.scale, h.cap) == (64, 0, 0, 0.125, 0.0)
    with pytest.raises(ValueError):
        X.make_heads(8, 2, 64, pairing="both")


# ---------------------------------------------------------------- the reference itself

def test_reference_gradients_match_differences():
    """The 64-bit reverse formulas against central differences of the forward: with a step s a difference is off by s^2
    / 6 times a third derivative (below 100 of the loss here) and 2^-52 / s of the loss by rounding."""
    g = torch.Generator().manual_seed(1)
    n = lambda *z: torch.randn(*z, generator=g, dtype=torch.float64)   # noqa: E731
    T, D, s = 7, 32, 1e-4
    q, k, v, go = n(T, D), n(T, D), n(T, D), n(T, D)
    lo, hi = U.spans(T, T, 0, [0, 4, 6], [2, 0])
    j = torch.arange(T)
    seen = (j[None] >= lo[:, None]) & (j[None] < hi[:, None])
    assert seen.sum(1).tolist() == [2, 2, 3, 4, 1, 2, 0]
    dist = (j[:, None] - j[None]).abs().double()
    args = lambda q, k, v: U.attention(q, k, v, seen, 0.3, 2.0, 0.1, dist, 0.0, go)   # noqa: E731
    r = args(q, k, v)
    assert bool((r["out"][0][6] == 0).all())
    loss = lambda *z: float((args(*z)["out"][0] * go).sum())   # noqa: E731
    for i, name in enumerate(("dq", "dk", "dv")):
        d = n(T, D)
        at = [q, k, v]
        plus, minus = list(at), list(at)
        plus[i], minus[i] = at[i] + s * d, at[i] - s * d
        diff = (loss(*plus) - loss(*minus)) / (2 * s)
        exact = float((r[name][0] * d).sum())
        assert abs(diff - exact) <= 1e-6 * float((r[name][0].abs() * d.abs()).sum()), name


def test_reference_codes():
    """What the cache holds: every value to within half the distance of its neighbours on the scale."""
    g = torch.Generator().manual_seed(2)
    x = torch.randn(50, 64, generator=g)
    h = U.held(x).view(50, 2, 32)
    y = x.double().view(50, 2, 32)
    top = y.abs().amax(-1, keepdim=True)
    assert bool(((h - y).abs() <= top / 6 * (1 + 2.0 ** -8) * torch.where(y.abs() > top / 1.5, 1.0, 0.5) + 1e-9).all())
    assert torch.equal(U.held(torch.zeros(1, 32)), torch.zeros(1, 32, dtype=torch.float64))
