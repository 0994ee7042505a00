"""The global gradient norm and clip on the GPU against 64 bits."""

import math

import pytest
import torch

from paper_2607_14530_amd import xhc as X

pytestmark = pytest.mark.gpu
F64 = torch.float64
BF, F32 = torch.bfloat16, torch.float32


def tensors(sizes, dtypes, seed, std=1.0, offset=0):
    """Tensors of the given sizes; offset: elements that their starts lie off 16 bytes."""
    g = torch.Generator().manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        t = dtypes[i % len(dtypes)]
        buf = (torch.randn(n + offset, generator=g) * std).to(t).cuda()
        out.append(buf[offset:])
    return out


def reference(grads, max_norm):
    total = math.fsum(float(g.cpu().to(F64).pow(2).sum()) for g in grads)
    norm = math.sqrt(total)
    return norm, min(1.0, max_norm / (norm + 1e-6))


def check(grads, max_norm, outs, norm, before):
    ref, c = reference(before, max_norm)
    # the norm is rounded to fp32 once, sums in fp64 differ by their order
    assert abs(float(norm) - ref) <= 2 ** -24 * ref * 1.001 + 1e-45
    for g, o in zip(before, outs):
        v = g.cpu().to(F64) * c
        # c and the product are rounded to fp32, a bf16 result once more
        tol = v.abs() * (2.1 * 2 ** -24 + (2 ** -8 if o.dtype == BF else 0)) + 1e-40
        assert bool(((o.cpu().to(F64) - v).abs() <= tol).all())


SETS = {
    "one": [1], "few": [3, 16, 4096, 7], "empty ones": [0, 5, 0, 1], "chunks": [8191, 8192, 8193, 70000, 1],
    "launches": [1 + 37 * (i % 11) for i in range(300)], "large": [9_000_001, 5, 4_000_000],
}


@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("dtypes", [(F32,), (BF,), (BF, F32)])
@pytest.mark.parametrize("name", list(SETS))
def test_clip(name, dtypes, offset):
    for max_norm in (0.5, 1e6):
        grads = tensors(SETS[name], dtypes, 5, offset=offset)
        before = [g.clone() for g in grads]
        outs = [torch.full_like(g, 7.0) for g in grads]
        norm = X.clip_grad_norm(grads, max_norm, outs=outs)
        check(grads, max_norm, outs, norm, before)
        for g, b in zip(grads, before):
            assert torch.equal(g, b)
        n2 = torch.empty(1, device="cuda")
        X.xhc_grad_norm(grads, n2, torch.empty(X.xhc_grad_workspace_bytes(len(grads)), dtype=torch.uint8, device="cuda"))
        assert torch.equal(n2, norm)
        assert torch.equal(X.clip_grad_norm(grads, max_norm), norm)       # in place
        for g, o in zip(grads, outs):
            assert torch.equal(g, o)
