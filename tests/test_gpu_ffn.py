"""The gated feed-forward block on the GPU against 64 bits: values within
derived bounds at odd and ragged sizes, rows and widths that end inside a tile."""

import pytest
import torch

from paper_2607_14530_amd import xhc as X
from tests.ffn_util import HALF, assert_within, ffn_backward, ffn_forward, ffn_inputs

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}

# T, C, H: one token, few tokens with large weights, ragged tokens, widths and hidden widths that end inside a block of 16, 32, 64 or a
# tile, more than one tile each way
SIZES = [(1, 32, 1), (20, 4096, 4160), (64, 2080, 8200), (1, 256, 683), (3, 96, 33), (16, 64, 64), (17, 160, 200), (37, 2112, 341), (64, 256, 1000),
         (65, 512, 129), (130, 352, 520), (200, 32, 48), (257, 384, 1030), (300, 1056, 96)]


def make(T, C, H, state, act, seed, train):
    x, dF, w = ffn_inputs(T, C, H, DT[state], seed)
    d = X.make_dims(T, 1, 1, 1, C, state=state)
    cls = X.TrainableFeedForward if train else X.FeedForward
    return x, dF, w, cls(d, H, {k: v.cuda() for k, v in w.items()}, act=act)


@pytest.mark.parametrize("state", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T,C,H", SIZES)
def test_forward_and_backward(T, C, H, state, act):
    x, dF, w, ff = make(T, C, H, state, act, 100 + T + C + H, True)
    F = ff.forward(x.cuda())
    dx = ff.backward(dF.cuda())
    torch.cuda.synchronize()
    half = HALF[DT[state]]
    fw = ffn_forward(x, w, act, half)
    assert_within(F, fw["F"], "F")
    bw = ffn_backward(x, dF, fw, act, half)
    assert_within(dx, bw["dx"], "dx")
    for n in ("W_gate", "W_up", "W_down"):
        assert_within(ff.grads[n], bw[n], "d" + n)


@pytest.mark.parametrize("state", ["bf16", "f32"])
@pytest.mark.parametrize("T,C,H", SIZES)
def test_forward_without_saving_gives_the_same(T, C, H, state):
    x, _, _, a = make(T, C, H, state, "silu", 7, False)
    _, _, _, b = make(T, C, H, state, "silu", 7, True)
    assert torch.equal(a.forward(x.cuda()), b.forward(x.cuda()))


@pytest.mark.parametrize("state,T,C,H", [("bf16", 1056, 1024, 8256), ("bf16", 1000, 2080, 4100), ("f32", 1030, 512, 8800)])
def test_large_tiles_and_a_rest_of_small_ones(state, T, C, H):
    """More than 256 large tiles, the last few computed as small ones."""
    x, dF, w, ff = make(T, C, H, state, "silu", 300 + T, True)
    F = ff.forward(x.cuda())
    dx = ff.backward(dF.cuda())
    torch.cuda.synchronize()
    half = HALF[DT[state]]
    fw = ffn_forward(x, w, "silu", half)
    assert_within(F, fw["F"], "F")
    bw = ffn_backward(x, dF, fw, "silu", half)
    assert_within(dx, bw["dx"], "dx")
    for n in ("W_gate", "W_up", "W_down"):
        assert_within(ff.grads[n], bw[n], "d" + n)


def check(T, C, H, state, seed):
    x, dF, w, ff = make(T, C, H, state, "silu", seed, True)
    F = ff.forward(x.cuda())
    dx = ff.backward(dF.cuda())
    torch.cuda.synchronize()
    half = HALF[DT[state]]
    fw = ffn_forward(x, w, "silu", half)
    assert_within(F, fw["F"], "F")
    bw = ffn_backward(x, dF, fw, "silu", half)
    assert_within(dx, bw["dx"], "dx")
    for n in ("W_gate", "W_up", "W_down"):
        assert_within(ff.grads[n], bw[n], "d" + n)


@pytest.mark.parametrize("state", ["bf16", "f32"])
@pytest.mark.parametrize("T", [16, 17, 32, 33, 48, 49, 64])
@pytest.mark.parametrize("C,H", [(64, 4160), (4128, 65), (224, 350)])
def test_few_tokens_with_many_and_few_blocks_of_weights(C, H, T, state):
    check(T, C, H, state, 400 + T)


def test_few_tokens_with_large_weights_and_an_fp32_state():
    check(61, 4128, 10700, "f32", 500)


@pytest.mark.parametrize("state", ["bf16", "f32"])
@pytest.mark.parametrize("T,C,H", [(97, 256, 683), (190, 544, 1311), (700, 320, 70), (1100, 96, 200)])
def test_short_products(T, C, H, state):
    check(T, C, H, state, 600 + T)
