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
    monkeypatch.setattr(X, "_settle", lambda: None)
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


BIG = [2 ** 31, 2 ** 32, 2 ** 32 + 5, -2 ** 31 - 1, -2 ** 32 + 64]


@pytest.mark.parametrize("v", BIG)
def test_heads_that_do_not_fit_their_fields_are_refused(v):
    """A field keeps 32 bits: a window of 2^32 + 5 would be one of 5."""
    for kw in (dict(Hq=v), dict(Hkv=v), dict(D=v), dict(rotary=v), dict(window=v)):
        with pytest.raises(ValueError):
            X.make_heads(**{**dict(Hq=4, Hkv=2, D=64, scale=0.125), **kw})
    assert X.make_heads(4, 2, 64, window=2 ** 31 - 1).window == 2 ** 31 - 1


@pytest.mark.parametrize("kw", [dict(sequences=65536, per_sequence=65537), dict(npages=2 ** 32 + 8), dict(page=2 ** 32 + 64),
                                dict(sequences=2 ** 32 + 2), dict(per_sequence=2 ** 32 + 2, npages=8)])
def test_caches_that_do_not_fit_their_fields_are_refused(calls, kw, monkeypatch):
    """A pool of 2^32 + 65536 pages would be one of 65536, and what lies in the others lost."""
    made = []
    monkeypatch.setattr(torch, "zeros", lambda *a, **k: made.append(a))
    h = X.make_heads(Hq, Hkv, D, rotary=0)
    with pytest.raises(ValueError):
        X.KVCache(X.make_dims(T, 1, 1, 1, 32), h, None, device="cpu", **{**dict(sequences=2, per_sequence=2, page=32), **kw})
    assert not made


@pytest.mark.parametrize("n", [2 ** 31, 2 ** 32 + 1])
def test_more_documents_than_their_number_holds_are_refused(calls, n):
    class Starts:
        dtype, shape = torch.int32, (n + 1,)
        numel = staticmethod(lambda: n + 1)
    with pytest.raises(ValueError):
        attention().spans(Starts)
    assert not calls
