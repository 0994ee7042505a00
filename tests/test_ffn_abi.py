"""The norm, the feed-forward block and the gradient clip refuse what they do
not take before any launch (no GPU needed: nothing below is dereferenced)."""

import ctypes

import pytest
import torch

from paper_2607_14530_amd import xhc as X
from tests import ffn_util as U

A = [(i + 1) << 24 for i in range(12)]       # distinct 16-byte aligned addresses
BIG = 1 << 50


def dims(**kw):
    base = dict(T=64, N=1, k=1, m=1, C=256)
    base.update(kw)
    return X.make_dims(**base)


def norm(d, p, **kw):
    q = dict(enumerate(p))
    q.update(kw)
    return X.lib().xhc_rmsnorm(ctypes.byref(d), *[q[i] for i in range(4)], None)


def norm_bwd(d, p, ws=BIG):
    return X.lib().xhc_rmsnorm_bwd(ctypes.byref(d), *p, ws, None)


def ffn(d, H, act, p, ws=BIG):
    return X.lib().xhc_ffn(ctypes.byref(d), H, act, *p, ws, None)


def ffn_bwd(d, H, act, p, ws=BIG):
    return X.lib().xhc_ffn_bwd(ctypes.byref(d), H, act, *p, ws, None)


def with_at(p, i, v):
    return [v if j == i else a for j, a in enumerate(p)]


def test_norm_refusals():
    d = dims()
    p = A[:4]                                 # x, gain, y, rstd
    for i in (0, 1, 2):
        assert norm(d, with_at(p, i, None)) == X.XHC_EINVAL
    for i in range(4):
        assert norm(d, with_at(p, i, p[i] + 4)) == X.XHC_EUNSUPPORTED
    for i, j in ((2, 0), (2, 1), (3, 0), (3, 1), (3, 2)):
        assert norm(d, with_at(p, i, p[j])) == X.XHC_EINVAL
    assert norm(dims(T=(1 << 23) + 1), p) == X.XHC_EUNSUPPORTED
    assert norm(dims(C=40), p) == X.XHC_EUNSUPPORTED
    assert norm(dims(eps=0.0), p) == X.XHC_EINVAL
    assert norm(dims(T=0, S=1), [None] * 4) == X.XHC_OK
    b = A[:7]                                 # x, gain, rstd, dy, dx, dgain, workspace
    for i in range(7):
        assert norm_bwd(d, with_at(b, i, None)) == X.XHC_EINVAL
        assert norm_bwd(d, with_at(b, i, b[i] + 8)) == X.XHC_EUNSUPPORTED
    for i in (0, 1, 2, 3):
        assert norm_bwd(d, with_at(b, 4, b[i])) == X.XHC_EINVAL
        assert norm_bwd(d, with_at(b, 5, b[i])) == X.XHC_EINVAL
    assert norm_bwd(d, with_at(b, 4, b[5])) == X.XHC_EINVAL
    need = X.xhc_rmsnorm_workspace_bytes(d)
    assert need > 0 and norm_bwd(d, b, need - 1) == X.XHC_EWORKSPACE


def test_ffn_refusals():
    d = dims()
    p = A[:5]                                 # input, packed, F, saved, workspace
    for i in (0, 1, 2, 4):
        assert ffn(d, 100, 0, with_at(p, i, None)) == X.XHC_EINVAL
    for i in range(5):
        assert ffn(d, 100, 0, with_at(p, i, p[i] + 2)) == X.XHC_EUNSUPPORTED
    for i, j in ((2, 0), (2, 1), (3, 0), (3, 1), (3, 2)):
        assert ffn(d, 100, 0, with_at(p, i, p[j])) == X.XHC_EINVAL
    for act in (-1, 2):
        assert ffn(d, 100, act, p) == X.XHC_EINVAL
    assert ffn(d, 0, 0, p) == X.XHC_EINVAL
    assert ffn(d, (1 << 20) + 1, 0, p) == X.XHC_EUNSUPPORTED
    assert ffn(dims(T=1 << 30), 4096, 0, p) == X.XHC_EUNSUPPORTED
    assert ffn(dims(C=48), 100, 0, p) == X.XHC_EUNSUPPORTED
    for dt in ("bf16", "f32"):
        e = dims(state=dt)
        assert ffn(e, 100, 0, p, X.xhc_ffn_workspace_bytes(e, 100, 0) - 1) == X.XHC_EWORKSPACE
    assert ffn(dims(T=0, S=1), 100, 0, [None] * 5) == X.XHC_OK
    b = A[:9]                                 # input, packed, saved, dF, d_input, dW_gate, dW_up, dW_down, workspace
    for i in range(9):
        assert ffn_bwd(d, 100, 0, with_at(b, i, None)) == X.XHC_EINVAL
        assert ffn_bwd(d, 100, 0, with_at(b, i, b[i] + 8)) == X.XHC_EUNSUPPORTED
    for out in (4, 5, 6, 7):
        for other in range(8):
            if other != out:
                assert ffn_bwd(d, 100, 0, with_at(b, out, b[other])) == X.XHC_EINVAL
    assert ffn_bwd(d, 100, 0, b, X.xhc_ffn_workspace_bytes(d, 100, 1) - 1) == X.XHC_EWORKSPACE


def test_ffn_sizes():
    d = dims(C=256)
    # K is laid out in blocks of 64: gate and up [256 x 2 128], down [128 x 256], twice with the backward's
    assert X.xhc_packed_ffn_bytes(d, 100, 0) == 256 * 256 * 2 + 128 * 256 * 2
    assert X.xhc_packed_ffn_bytes(d, 100, 1) == 2 * X.xhc_packed_ffn_bytes(d, 100, 0)
    assert X.xhc_ffn_saved_bytes(d, 100) == 2 * 64 * 128 * 3
    assert X.xhc_ffn_saved_bytes(dims(state="f32"), 100) == 2 * 64 * 128 * 4
    assert X.xhc_packed_ffn_bytes(d, 0, 1) == 0 and X.xhc_ffn_workspace_bytes(d, 1 << 21, 1) == 0
    assert X.lib().xhc_pack_ffn(ctypes.byref(d), 100, A[0], A[1], None, 1, A[3], None) == X.XHC_EINVAL
    assert X.lib().xhc_pack_ffn(ctypes.byref(d), 100, A[0], A[1], A[2], 2, A[3], None) == X.XHC_EINVAL
    assert X.lib().xhc_pack_ffn(ctypes.byref(d), 100, A[0], A[1], A[2], 1, A[2], None) == X.XHC_EINVAL
    assert X.lib().xhc_pack_ffn(ctypes.byref(d), 100, A[0] + 4, A[1], A[2], 1, A[3], None) == X.XHC_EUNSUPPORTED


def clip(tensors, max_norm=1.0, ws=BIG, norm=A[11], work=A[10], n=None):
    """tensors: (grad, count, dtype, out)"""
    m = len(tensors)
    g, c, t, o = zip(*tensors) if tensors else ((), (), (), ())
    return X.lib().xhc_grad_clip(m if n is None else n, (ctypes.c_void_p * m)(*g), (ctypes.c_int64 * m)(*c),
                                 (ctypes.c_int32 * m)(*t), max_norm, (ctypes.c_void_p * m)(*o), norm, work, ws, None)


F, B = X.XHC_F32, X.XHC_BF16


@pytest.mark.parametrize("tensors,status", [
    ([(A[0], 10, 2, A[0])], X.XHC_EINVAL),                               # dtype
    ([(A[0], -1, F, A[0])], X.XHC_EINVAL),                               # count
    ([(None, 4, F, A[0])], X.XHC_EINVAL),
    ([(A[0], 4, F, None)], X.XHC_EINVAL),
    ([(A[0] + 2, 4, F, A[1])], X.XHC_EUNSUPPORTED),                      # not on an element
    ([(A[0], 4, B, A[1] + 1)], X.XHC_EUNSUPPORTED),
    ([(A[0], (1 << 40) + 1, B, A[0])], X.XHC_EUNSUPPORTED),
    ([(A[0], 1 << 39, B, A[0]), (1 << 55, 1 << 39, B, 1 << 55), (1 << 56, 1, F, 1 << 56)], X.XHC_EUNSUPPORTED),
    ([(A[0], 8, F, A[0]), (A[0], 8, F, A[0])], X.XHC_EINVAL),            # the same tensor twice, in place
    ([(A[0], 8, F, A[1]), (A[0] + 4, 8, F, A[1] + 28)], X.XHC_EINVAL),   # outputs overlap
    ([(A[0], 8, F, A[0] + 16)], X.XHC_EINVAL),                           # an output overlaps its gradient
    ([(A[0], 8, F, A[1]), (A[1] + 31, 1, B, A[2])], X.XHC_EUNSUPPORTED),
    ([(A[0], 8, F, A[1]), (A[1] + 30, 1, B, A[2])], X.XHC_EINVAL),       # an output overlaps another gradient
    ([(A[11] - 4, 2, F, A[11] - 4)], X.XHC_EINVAL),                      # the norm inside an output
])
def test_clip_refusals(tensors, status):
    assert clip(tensors) == status


def test_clip_refusals_of_the_call():
    one = [(A[0], 8, F, A[0])]
    for bad in (-1.0, float("nan")):
        assert clip(one, max_norm=bad) == X.XHC_EINVAL
    assert clip(one, n=-1) == X.XHC_EINVAL
    assert clip(one, norm=None) == X.XHC_EINVAL
    assert clip(one, work=None) == X.XHC_EINVAL
    assert clip(one, norm=A[11] + 2) == X.XHC_EUNSUPPORTED
    assert clip(one, ws=X.xhc_grad_workspace_bytes(1) - 1) == X.XHC_EWORKSPACE
    many = [(A[0] + 64 * i, 1, F, A[0] + 64 * i) for i in range(4097)]
    assert clip(many) == X.XHC_EUNSUPPORTED
    assert X.xhc_grad_workspace_bytes(4097) == 0 and X.xhc_grad_workspace_bytes(-1) == 0
    assert X.lib().xhc_grad_norm(1, None, None, None, A[11], A[10], BIG, None) == X.XHC_EINVAL


def test_binding_refusals():
    with pytest.raises(ValueError):
        X.xhc_grad_norm([torch.zeros(4, dtype=torch.float16)], None, None)
    with pytest.raises(ValueError):
        X.xhc_grad_norm([torch.zeros(4)], None, None)                    # not on a GPU
    assert [tuple(t.shape) for t in X.grad_tensors(
        [{"X": torch.zeros(9), "F": torch.zeros(9), "dp": torch.zeros(9), "W_r": torch.zeros(2), "conv_w": None},
         {"F_list": [torch.zeros(9)], "b_post": [torch.zeros(3), torch.zeros(4)]}, {"gain": torch.zeros(5)}])] \
        == [(2,), (3,), (4,), (5,)]


# ---------------------------------------------------------------- the reference itself

@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_reference_gradients_match_differences(kind):
    """The 64-bit reverse formulas against central differences of the forward:
    with a step s the difference is off by s^2 / 6 times a third derivative
    (below 20 of the loss here) and 2^-52 / s of the loss by rounding."""
    T, C, H, s = 3, 32, 5, 1e-4
    g = torch.Generator().manual_seed(3)
    n = lambda *z: torch.randn(*z, generator=g, dtype=torch.float64)   # noqa: E731
    x, dF, Wg, Wu, Wd = n(T, C), n(T, C), n(C, H) * C ** -0.5, n(C, H) * C ** -0.5, n(H, C)

    def loss(x, Wg, Wu, Wd):
        return float(((U.act(x @ Wg, kind)[0] * (x @ Wu)) @ Wd * dF).sum())

    a, da = U.act(x @ Wg, kind)
    fw = dict(g=(x @ Wg, 0 * a), u=(x @ Wu, 0 * a), a=a, da=da, W=(Wg, Wu, Wd))
    bw = U.ffn_backward(x, dF, fw, kind, U.HALF[torch.float32])
    args = [x, Wg, Wu, Wd]
    for i, name in enumerate(("dx", "W_gate", "W_up", "W_down")):
        d = n(*args[i].shape)
        plus, minus = list(args), list(args)
        plus[i], minus[i] = args[i] + s * d, args[i] - s * d
        diff = (loss(*plus) - loss(*minus)) / (2 * s)
        exact = float((bw[name][0] * d).sum())
        size = float((bw[name][0].abs() * d.abs()).sum())
        assert abs(diff - exact) <= 1e-6 * size, (name, diff, exact)
    # the norm
    w = 1 + 0.1 * n(C)
    (dx, _), (dw, _) = U.norm_backward(x, w, dF, 1e-5, 0.0)
    f = lambda x, w: float((U.norm_forward(x, w, 1e-5, 0.0)[0] * dF).sum())   # noqa: E731
    for v, grad, at in ((n(T, C), dx, 0), (n(C), dw, 1)):
        p = [x + s * v, w] if at == 0 else [x, w + s * v]
        m = [x - s * v, w] if at == 0 else [x, w - s * v]
        assert abs((f(*p) - f(*m)) / (2 * s) - float((grad * v).sum())) <= 1e-6 * float((grad.abs() * v.abs()).sum())
