"""What the bundles of the norm and the feed-forward block hand to the C entry
points, with those replaced by a record (no GPU needed)."""

from types import SimpleNamespace

import pytest
import torch

from paper_2607_14530_amd import xhc as X

T, C, H = 6, 32, 5
BF = torch.bfloat16


@pytest.fixture
def calls(monkeypatch):
    made = []
    for name in ("xhc_rmsnorm", "xhc_rmsnorm_bwd", "xhc_ffn", "xhc_ffn_bwd", "xhc_pack_ffn"):
        def record(*args, name=name):
            if any(torch.is_tensor(a) and a.numel() and not a.is_contiguous() for a in args):
                raise ValueError("tensor arguments must be contiguous")
            made.append((name, args))
        monkeypatch.setattr(X, name, record)
    monkeypatch.setattr(X, "_here", lambda device: torch.device("cpu"))
    return made


def norm():
    return X.TrainableRMSNorm(X.make_dims(T, 1, 1, 1, C), torch.ones(C), "cpu")


def block():
    w = {"W_gate": torch.ones(C, H), "W_up": torch.ones(C, H), "W_down": torch.ones(H, C)}
    return X.TrainableFeedForward(X.make_dims(T, 1, 1, 1, C), H, w, device="cpu")


@pytest.mark.parametrize("make,back,at", [(norm, "xhc_rmsnorm_bwd", 1), (block, "xhc_ffn_bwd", 3)])
def test_a_refused_forward_leaves_the_last_ones_input(calls, make, back, at):
    """The backward reads the input of the last forward that ran, never one that was refused."""
    f, x, dy = make(), torch.zeros(T, C, dtype=BF), torch.zeros(T, C, dtype=BF)
    bad = [x[:2], x.float(), torch.zeros(C, T, dtype=BF).t(), torch.zeros(T, C, dtype=BF, device="meta")]
    for b in bad:
        with pytest.raises(ValueError):
            f.forward(b)
        with pytest.raises(ValueError):
            f.backward(dy)                    # no forward has run
    f.forward(x)
    for b in bad:
        with pytest.raises(ValueError):
            f.forward(b)
        f.backward(dy)
        assert calls[-1][0] == back and calls[-1][1][at] is x


@pytest.mark.parametrize("make", [norm, block])
def test_a_call_while_another_device_is_current_is_refused(calls, make, monkeypatch):
    """Launches go to the current device: it has to be the one that holds the bundle's buffers."""
    f, there = make(), torch.device("cuda", 1)
    x = SimpleNamespace(dtype=BF, shape=(T, C), device=there, is_cuda=True, is_contiguous=lambda: True)
    f.device = there
    current = [1]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    f.forward(x)
    f.backward(x)
    current[0] = 0
    made = len(calls)
    for call in (f.forward, f.backward):
        with pytest.raises(ValueError, match="current device"):
            call(x)
    if make is block:
        with pytest.raises(ValueError, match="current device"):
            f.pack({"W_gate": torch.ones(C, H), "W_up": torch.ones(C, H), "W_down": torch.ones(H, C)})
    assert len(calls) == made
