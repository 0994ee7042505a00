"""A new bundle's first call on another stream than the one it was made on, which
still has work in the memory that the bundle's buffers were given."""

import pytest
import torch

from paper_2607_14530_amd import xhc as X
from tests import attn_util as U

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
T, Hq, Hkv, D = 1024, 8, 2, 64


def work_in_freed_memory(sizes):
    """Long work on the current stream whose last steps write to memory of these sizes, which is free already."""
    busy = torch.randn(4096, 4096, device="cuda")
    old = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
    torch.cuda.synchronize()
    for _ in range(20):
        busy = busy @ busy * 1e-2
    for t in old:
        t.fill_(77)


def test_a_first_step_on_another_stream():
    d, h = X.make_dims(T, 1, 1, 1, 32, S=T), X.make_heads(Hq, Hkv, D)
    qkv, dout = (z.cuda() for z in U.inputs(T, Hq, Hkv, D, BF, 1))
    ref = X.TrainableAttention(d, h)
    out, grad = ref.forward(qkv).clone(), ref.backward(dout).clone()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    work_in_freed_memory([t.numel() * t.element_size() for t in (ref.out, ref.saved, ref.dqkv, ref.ws)])
    att = X.TrainableAttention(d, h)
    att.forward(qkv, stream=s)
    att.backward(dout, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(att.out, out) and torch.equal(att.dqkv, grad)


def test_a_first_prompt_on_another_stream():
    d, h = X.make_dims(T, 1, 1, 1, 32, S=T), X.make_heads(Hq, Hkv, D)
    qkv, _ = (z.cuda() for z in U.inputs(T, Hq, Hkv, D, BF, 2))
    table = X.rotation_table(T, D)
    rot = X.Rotation(d, h, table)
    ref = X.Attention(d, h)
    x0 = rot.forward(qkv).clone()
    out = ref.forward(x0).clone()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    work_in_freed_memory([t.numel() * t.element_size() for t in (ref.out, x0)])
    rot2, att = X.Rotation(d, h, table), X.Attention(d, h)
    x = rot2.forward(qkv, stream=s)
    y = att.forward(x, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(x, x0) and torch.equal(y, out)
