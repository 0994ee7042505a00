"""The gradient norm and clip at the borders of their tables and workspaces."""

import pytest
import torch

from paper_2607_14530_amd import xhc as X

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("q", [8192, 10240])
def test_the_workspace_of_the_query_is_enough(q):
    """A total just below the next multiple of the number of chunks, in one
    tensor: nothing is written behind the workspace that the query names."""
    n = 16384 * q + 16383
    g = torch.full((n,), 2.0 ** -10, dtype=BF, device="cuda")
    need = X.xhc_grad_workspace_bytes(1)
    buf = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    norm = torch.empty(1, device="cuda")
    ref = (n ** 0.5) * 2.0 ** -10
    for out in (None, torch.empty_like(g)):
        if out is None:
            X.xhc_grad_norm([g], norm, buf[:need])
        else:
            X.xhc_grad_clip([g], 0.5, [out], norm, buf[:need])
        torch.cuda.synchronize()
        assert bool((buf[need:] == 0xA5).all())
        # squares and their sums (below 2^53 times the smallest) are exact in fp64; one rounding to fp32
        assert abs(float(norm) - ref) <= 2.0 ** -24 * ref * 1.001
    # c and the product are rounded to fp32, the output to bf16: one value throughout
    v = 0.5 / (ref + 1e-6) * 2.0 ** -10
    assert bool((out == out[0]).all())
    assert abs(float(out[0]) - v) <= v * (2.0 ** -8 + 2.1 * 2.0 ** -24)
