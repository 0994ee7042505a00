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


def block(T, C, H):
    d = X.make_dims(T, 1, 1, 1, C)
    back = X.lib().xhc_ffn_bwd(ctypes.byref(d), H, 0, *A[:9], BIG, None)
    return X.lib().xhc_ffn(ctypes.byref(d), H, 0, *A[:5], BIG, None), back, X.xhc_ffn_workspace_bytes(d, H, 1) > 0


# the rows are brought into fragments by a wave each: T in whole blocks of 16, C in blocks of 64, 8 elements a thread
@pytest.mark.parametrize("T,C,H,fits", [
    ((1 << 29) - 32, 32, 16, True), ((1 << 29) - 16, 32, 16, False), ((1 << 29) - 31, 32, 1, False),
    (1 << 29, 32, 1, False), (1 << 28, 64, 32, True), ((1 << 28) + 1, 64, 32, False),
    (1 << 14, 1 << 20, 8192, True), (1 << 13, 8192, 1 << 20, True), (1, 32, (1 << 20) + 1, False)])
def test_block(T, C, H, fits):
    assert block(T, C, H) == ((OK, OK, True) if fits else (X.XHC_EUNSUPPORTED,) * 2 + (False,))
