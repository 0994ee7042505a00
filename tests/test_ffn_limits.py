"""Sizes past what a launch takes are refused, those just below are not
(checked up to the first launch, which fails without a GPU)."""

import ctypes

import pytest
import torch

from paper_2607_14530_amd import xhc as X

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: runs where no launch can happen")

A = [(i + 1) << 44 for i in range(12)]       # distinct 16-byte aligned addresses
BIG = 1 << 62
OK = X.XHC_EHIP                              # accepted: the launch itself fails here


def norm(T, C):
    d = X.make_dims(T, 1, 1, 1, C)
    back = X.lib().xhc_rmsnorm_bwd(ctypes.byref(d), *A[:7], BIG, None)
    return X.lib().xhc_rmsnorm(ctypes.byref(d), *A[:4], None), back, X.xhc_rmsnorm_workspace_bytes(d) > 0


@pytest.mark.parametrize("T,C,fits", [
    (1, 1 << 27, True), (1, (1 << 27) + 32, False), (1, (1 << 31) - 32, False),
    (1 << 23, 4096, True), ((1 << 23) + 1, 32, False)])
def test_norm(T, C, fits):
    assert norm(T, C) == ((OK, OK, True) if fits else (X.XHC_EUNSUPPORTED,) * 2 + (False,))
