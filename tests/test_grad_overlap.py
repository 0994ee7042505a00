"""A clip refuses outputs, and a norm, that lie in its workspace (made-up
addresses, nothing is dereferenced before the refusal)."""

import ctypes

import pytest
import torch

from paper_2607_14530_amd import xhc as X

G, O, W, N = [(i + 1) << 24 for i in range(4)]
BIG = 1 << 50


def clip(grad, out, norm, count=64):
    need = X.xhc_grad_workspace_bytes(1)
    assert need % 8 == 0
    a = lambda t, v: (t * 1)(v)   # noqa: E731
    return X.lib().xhc_grad_clip(1, a(ctypes.c_void_p, grad), a(ctypes.c_int64, count), a(ctypes.c_int32, X.XHC_F32), 1.0,
                                 a(ctypes.c_void_p, out), norm, W, BIG, None)


def test_workspace_overlap():
    need = X.xhc_grad_workspace_bytes(1)
    for at in (W, W + need - 16, W - 240):
        assert clip(G, at, N) == X.XHC_EINVAL            # an output
        assert clip(at, at, N) == X.XHC_EINVAL           # a gradient in place
        assert clip(at, O, N) == X.XHC_EINVAL            # a gradient: the sums would be written over it
    for at in (W, W + need - 4):
        assert clip(G, O, at) == X.XHC_EINVAL            # the norm


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: runs where no launch can happen")
def test_beside_the_workspace():
    need = X.xhc_grad_workspace_bytes(1)
    for at in (W + need, W - 256):
        assert clip(G, at, N) == X.XHC_EHIP              # accepted: the launch itself fails here
    assert clip(G, O, W + need) == X.XHC_EHIP
