"""A training step of a stack of xHC sublayers with the library's own norm and
feed-forward block as the sublayers' function, and the clip of all gradients:
each part against 64 bits from the inputs that it had on the GPU."""

import math

import pytest
import torch

from paper_2607_14530_amd import synth
from paper_2607_14530_amd import xhc as X
from tests.ffn_util import HALF, assert_within, ffn_backward, ffn_forward, norm_backward, norm_forward

pytestmark = pytest.mark.gpu
F64 = torch.float64


@pytest.mark.parametrize("state", ["bf16", "f32"])
def test_stack_with_norm_block_and_clip(state):
    T, S, N, k, m, C, H = 96, 48, 8, 4, 2, 256, 340
    dt = torch.bfloat16 if state == "bf16" else torch.float32
    half = HALF[dt]
    subs, norms, blocks, weights, gains, inputs = [], [], [], [], [], []
    for l, Kr in enumerate((4, 4)):
        w = synth.Workload(T=T, S=S, N=N, k=k, m=m, C=C, Kr=Kr, state=state, alpha=(0.1, 0.5, 0.1), name=f"mlp-{l}")
        inp = synth.sublayer_inputs(w, 150 + l, device="cuda")
        if l == 0:
            x0 = inp["X"].clone()
        d = X.dims_for(w)
        g = torch.Generator().manual_seed(160 + l)
        ffw = {"W_gate": torch.randn(C, H, generator=g) * C ** -0.5, "W_up": torch.randn(C, H, generator=g) * C ** -0.5,
               "W_down": torch.randn(H, C, generator=g) * H ** -0.5}
        gain = 1 + 0.1 * torch.randn(C, generator=g)
        subs.append(X.TrainableSublayer(d, inp, "cuda"))
        norms.append(X.TrainableRMSNorm(d, gain.cuda()))
        blocks.append(X.TrainableFeedForward(d, H, {n: v.cuda() for n, v in ffw.items()}))
        weights.append(ffw)
        gains.append(gain)
    fns = [lambda x, l=l: blocks[l].forward(norms[l].forward(x)) for l in range(2)]
    dFs = {}

    def back(l, dF):
        dFs[l] = dF.clone()
        return norms[l].backward(blocks[l].backward(dF))

    stack = X.Stack(subs)
    state_x = x0.clone()
    stack.forward(state_x, fns)
    inputs = [s.input.clone() for s in subs]
    G = torch.randn(T, C, generator=torch.Generator().manual_seed(170)).to(dt).cuda()
    grads, _ = stack.backward(state_x, G, [lambda dF, l=l: back(l, dF) for l in range(2)])
    torch.cuda.synchronize()
    assert torch.equal(state_x, x0)
    eps = subs[0].d.eps
    for l in range(2):
        x, y = inputs[l].cpu(), norms[l].y.cpu()
        ry, ey, _, _ = norm_forward(x, gains[l], eps, half)
        assert_within(y, (ry, ey), "norm")
        fw = ffn_forward(y, weights[l], "silu", half)
        assert_within(stack.F[l], fw["F"], "block")
        bw = ffn_backward(y, dFs[l].cpu(), fw, "silu", half)
        assert_within(blocks[l].d_input, bw["dx"], "block's input gradient")
        for n in weights[l]:
            assert_within(blocks[l].grads[n], bw[n], "d" + n)
        (dx, ex), dw = norm_backward(x, gains[l], blocks[l].d_input.cpu(), eps, half)
        assert_within(norms[l].dx, (dx, ex), "norm's input gradient")
        assert_within(norms[l].grads["gain"], dw, "dgain")
    # the connection's fp32 gradients and the block's in one clip
    every = X.grad_tensors([grads, [b.grads for b in blocks], [n.grads for n in norms]])
    assert len(every) == 2 * (9 + 3 + 1)
    before = [t.clone() for t in every]
    ref = math.sqrt(math.fsum(float(t.cpu().to(F64).pow(2).sum()) for t in before))
    norm = X.clip_grad_norm(every, 0.25)
    assert abs(float(norm) - ref) <= 2.0 ** -23 * ref
    c = min(1.0, 0.25 / (ref + 1e-6))
    assert c < 1.0
    for t, b in zip(every, before):
        v = b.cpu().to(F64) * c
        # c and the product rounded to fp32, a bf16 gradient once more
        tol = v.abs() * (3 * 2.0 ** -24 + (2.0 ** -8 if t.dtype == torch.bfloat16 else 0)) + 1e-40
        assert bool(((t.cpu().to(F64) - v).abs() <= tol).all())
