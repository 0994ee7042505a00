"""RMSNorm on the GPU against 64 bits, within derived bounds."""

import pytest
import torch

from paper_2607_14530_amd import xhc as X
from tests.ffn_util import HALF, assert_within, norm_backward, norm_forward

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
# widths of one to eight vectors per lane with full and ragged last ones, and wider than a wave holds
SIZES = [(1, 32), (3, 4096), (5, 96), (63, 512), (64, 544), (65, 1024), (129, 1056), (777, 2112), (40, 4064),
         (9, 4128), (70, 8192), (2100, 64)]


@pytest.mark.parametrize("state", ["bf16", "f32"])
@pytest.mark.parametrize("T,C", SIZES)
def test_forward_and_backward(T, C, state):
    g = torch.Generator().manual_seed(T + C)
    x = (torch.randn(T, C, generator=g) * torch.exp(torch.randn(T, 1, generator=g) * 2)).to(DT[state])
    dy = torch.randn(T, C, generator=g).to(DT[state])
    gain = 1 + 0.2 * torch.randn(C, generator=g)
    d = X.make_dims(T, 1, 1, 1, C, state=state, eps=1e-5)
    nm = X.TrainableRMSNorm(d, gain.cuda())
    y = nm.forward(x.cuda())
    dx = nm.backward(dy.cuda())
    torch.cuda.synchronize()
    half = HALF[DT[state]]
    ry, ey, r, rel = norm_forward(x, gain, 1e-5, half)
    assert_within(y, (ry, ey), "y")
    assert_within(nm.rstd, (r[:, 0], (rel + 2 ** -22) * r[:, 0]), "rstd")
    rdx, rdw = norm_backward(x, gain, dy, 1e-5, half)
    assert_within(dx, rdx, "dx")
    assert_within(nm.grads["gain"], rdw, "dgain")
    assert torch.equal(X.RMSNorm(d, gain.cuda()).forward(x.cuda()), y)
