"""What the cache's bundle answers for tokens that no sequence has, or that are
not stored: what an earlier call left there, zeros at first."""

import pytest
import torch

from paper_2607_14530_amd import xhc as X

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
NAME = {BF: "bf16", F32: "f32"}
Hq, Hkv, D, PAGE = 4, 2, 64, 32


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def cache(T, B, per, dtype=BF, **kw):
    d = X.make_dims(T, 1, 1, 1, 32, S=1, state=NAME[dtype])
    return X.KVCache(d, X.make_heads(Hq, Hkv, D), X.rotation_table(per * PAGE, D), B, per, page=PAGE, **kw)


def leave_nan(T, dtype):
    """Freed memory of the bundle's buffers' sizes, full of NaN."""
    held = [torch.full((T, n, D), float("nan"), dtype=dtype, device="cuda") for n in (Hq, Hkv) for _ in range(6)]
    torch.cuda.synchronize()
    del held


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_of_no_sequence_are_zeros_at_first(dtype):
    """A padded batch: room for 40 tokens, of which the call has three, one of them past its sequence's table."""
    T, B = 40, 2
    leave_nan(T, dtype)
    c = cache(T, B, 2, dtype)
    qkv = torch.randn(T, Hq + 2 * Hkv, D, device="cuda").to(dtype)
    args = (i32([1, 3, 4]), i32([2, 2 * PAGE + 1]), i32([[0, 1], [2, 3]]))
    q = c.append(qkv, *args)
    out = c.attend(q, *args)
    k, v = c.read(*args)
    rest = [t for t in range(T) if t not in (1, 2)]
    for z in (q, out, k, v):
        assert bool((z[rest] == 0).all()) and bool((z[1:3] != 0).any(-1).all())
    # another call leaves the rows that it has no token for
    before = [z.clone() for z in (q, out, k, v)]
    args = (i32([7, 8, 8]), i32([3, 0]), i32([[0, 1], [2, 3]]))
    q = c.append(qkv, *args)
    got = (q, c.attend(q, *args), *c.read(*args))
    for z, b in zip(got, before):
        b[7] = z[7]
        assert torch.equal(z, b) and bool((z[7] != 0).any())


def test_a_captured_first_read_leaves_other_tokens():
    """The call that reads first is a captured one: replays answer for the tokens that they have."""
    T, B = 6, 1
    c = cache(T, B, 1)
    qkv = torch.randn(T, Hq + 2 * Hkv, D, device="cuda").to(BF)
    starts, lens, pages = i32([0, 6]), i32([6]), i32([[0]])
    c.append(qkv, starts, lens, pages)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        k, v = c.read(starts, lens, pages)
    g.replay()
    torch.cuda.synchronize()
    k0, v0 = k.clone(), v.clone()
    assert bool((k0 != 0).any(-1).all()) and bool((v0 != 0).any(-1).all())
    starts.copy_(i32([0, 2]))
    lens.copy_(i32([2]))
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(k, k0) and torch.equal(v, v0)
        k2, v2 = c.read(starts, lens, pages)
        assert k2 is k and v2 is v and torch.equal(k, k0)


def test_a_new_bundle_is_ready_for_any_stream():
    """Its buffers are filled when it is there: a first call on another stream is not overwritten."""
    T, B, per = 2048, 1, 64
    qkv = torch.randn(T, Hq + 2 * Hkv, D, device="cuda").to(BF)
    args = (i32([0, T]), i32([T]), torch.arange(per, device="cuda").int().view(1, per))
    want = cache(T, B, per)
    q0 = want.append(qkv, *args).clone()
    out0 = want.attend(q0, *args).clone()
    s = torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    for _ in range(20):
        busy = busy @ busy * 1e-2                # the current stream has work in front of the bundle's filling
    c = cache(T, B, per)
    q = c.append(qkv, *args, stream=s)
    out = c.attend(q, *args, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(q, q0) and torch.equal(out, out0)


@pytest.mark.parametrize("B", [3, 70])
def test_starts_that_do_not_ascend_stay_within_the_buffers(B):
    """Undefined outputs, but of the call's tokens only, and nothing of its workspace's surroundings is read as a sum
    of theirs: a token in front of the start of the sequence that the search finds is left to others."""
    T, per = 8, 64
    c = cache(T, B, per)
    n = c.ws.numel()
    around = torch.full((n + 8192,), 255, dtype=torch.uint8, device="cuda")
    assert around.data_ptr() % 16 == 0
    c.ws = around[4096:4096 + n]
    out = torch.full((T + 64, Hq, D), 7.0, dtype=BF, device="cuda")
    c.out = out[32:32 + T]
    starts, lens = [5, 6, 2] + [8] * (B - 2), [per * PAGE] * B
    pages = torch.arange(B * per, device="cuda").int().view(B, per)
    q = torch.randn(T, Hq, D, device="cuda").to(BF)
    c.attend(q, i32(starts), i32(lens), pages)
    torch.cuda.synchronize()
    assert bool((around[:4096] == 255).all()) and bool((around[4096 + n:] == 255).all())
    assert bool((out[:32] == 7).all()) and bool((out[32 + T:] == 7).all())
    assert bool(torch.isfinite(c.out.float()).all())           # (the pool holds zeros)
