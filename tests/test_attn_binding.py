"""What the attention's and the cache's bundles do on the host, with the C entry
points replaced by a record (no GPU needed)."""

import pytest
import torch

from paper_2607_14530_amd import xhc as X

BF = torch.bfloat16
T, Hq, Hkv, D = 6, 4, 2, 32


@pytest.fixture
def calls(monkeypatch):
    made = []
    for name in ("xhc_attn", "xhc_attn_bwd", "xhc_attn_spans", "xhc_rotate"):
        monkeypatch.setattr(X, name, lambda *args, name=name: made.append((name, args)))

    def take(t, dtype, shape, dev, name):
        X._expect(t, dtype, shape, name)
        return t
    monkeypatch.setattr(X, "_take", take)
    monkeypatch.setattr(X, "_here", lambda device: torch.device("cpu"))
    return made


def attention(cls=X.TrainableAttention):
    return cls(X.make_dims(T, 1, 1, 1, 32, S=T), X.make_heads(Hq, Hkv, D), device="cpu")


def qkv():
    return torch.zeros(T, Hq + 2 * Hkv, D, dtype=BF)


@pytest.mark.parametrize("change", [lambda o: o.mul_(2), lambda o: o.view(T, -1).add_(1), lambda o: o[2:3].zero_(),
                                    lambda o: torch.add(o, 1, out=o)])
def test_a_backward_after_a_change_of_the_returned_output_is_refused(calls, change):
    """The backward reads it again."""
    att, dout = attention(), torch.zeros(T, Hq, D, dtype=BF)
    out = att.forward(qkv())
    att.backward(dout)
    change(out)
    with pytest.raises(ValueError, match="output"):
        att.backward(dout)
    assert calls[-1][0] == "xhc_attn_bwd" and len(calls) == 2
    att.forward(qkv())                           # which writes it anew
    att.backward(dout)
    out * 2                                      # reading it is no change
    att.backward(dout)


def test_bundles_without_versions(calls):
    """Tensors made in inference mode have none."""
    with torch.inference_mode():
        att = attention()
        out = att.forward(qkv())
        att.backward(torch.zeros_like(out))
    assert [n for n, _ in calls] == ["xhc_attn", "xhc_attn_bwd"]
    att.forward(qkv())
    att.backward(torch.zeros(T, Hq, D, dtype=BF))


def test_a_refused_forward_leaves_the_last_ones_input(calls):
    att, x = attention(), qkv()
    with pytest.raises(ValueError):
        att.forward(x[:2])
    with pytest.raises(ValueError, match="without a forward"):
        att.backward(torch.zeros(T, Hq, D, dtype=BF))
    att.forward(x)
    for bad in (x[:2], x.float()):
        with pytest.raises(ValueError):
            att.forward(bad)
        att.backward(torch.zeros(T, Hq, D, dtype=BF))
        assert calls[-1][1][2] is x


def test_the_current_stream_by_public_names(monkeypatch):
    """A torch without the short way to a stream's handle has the documented one."""
    class Stream:
        cuda_stream = 1234
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream)
    assert X._stream(None) == 1234
    assert X._stream(Stream) == 1234 and X._stream(77) == 77
