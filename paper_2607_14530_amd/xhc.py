"""Python binding of libxhc.so (ctypes): argument marshalling only.

Every function named like a C entry point (xhc_pre, xhc_post, ...) takes the
same arguments as in include/xhc.h, with torch CUDA tensors in place of device
pointers; the stream defaults to torch's current stream.  All computation
runs in the library's HIP kernels.  There is no CPU fallback: if the library
is missing or no GPU is present, calls raise.

``Sublayer`` / ``FlashGroup`` bundle packing, output allocation and the calls
for convenience; they add no arithmetic.  ``RMSNorm`` and ``FeedForward`` (and
their trainable forms, whose forward and backward ``Stack`` takes as a
sublayer's functions) do the same for an MLP-type sublayer's own function, and
``clip_grad_norm`` for the clip of the gradients that a backward has given.
``Rotation``, ``Attention`` and ``TrainableAttention`` are an attention-type
sublayer's own function between its projections, ``KVCache`` its serving form:
a paged cache in 4 bits and the attention over it.
"""

from __future__ import annotations

import contextlib
import ctypes
import os
import re

import torch

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libxhc.so")
HEADER = os.path.join(os.path.dirname(PKG), "include", "xhc.h")

XHC_OK, XHC_EINVAL, XHC_EUNSUPPORTED, XHC_EWORKSPACE, XHC_EHIP = range(5)
STATUS_NAMES = {0: "XHC_OK", 1: "XHC_EINVAL", 2: "XHC_EUNSUPPORTED", 3: "XHC_EWORKSPACE", 4: "XHC_EHIP"}
XHC_BF16, XHC_F32 = 0, 1
XHC_IMPL_AUTO, XHC_IMPL_MULTI, XHC_IMPL_FUSED = 0, 1, 2
XHC_ROUTER_SIGMOID, XHC_ROUTER_SOFTMAX = 0, 1
XHC_ACT_SILU, XHC_ACT_GELU = 0, 1
XHC_PAIRS_HALVES, XHC_PAIRS_NEIGHBOURS = 0, 1
(XHC_OP_PRE, XHC_OP_POST, XHC_OP_FLASH_PRE, XHC_OP_FLASH_POST, XHC_OP_POST_BWD, XHC_OP_PRE_BWD,
 XHC_OP_FLASH_POST_BWD, XHC_OP_FLASH_PRE_BWD) = range(8)


class XhcError(RuntimeError):
    def __init__(self, name, status, detail=""):
        super().__init__(f"{name} returned {STATUS_NAMES.get(status, status)}{detail}")
        self.status = status


class Dims(ctypes.Structure):
    _fields_ = [
        ("T", ctypes.c_int64), ("S", ctypes.c_int64),
        ("N", ctypes.c_int32), ("k", ctypes.c_int32), ("m", ctypes.c_int32), ("C", ctypes.c_int32),
        ("Kr", ctypes.c_int32), ("kappa", ctypes.c_int32 * 3),
        ("sinkhorn_iters", ctypes.c_int32), ("gram_schmidt", ctypes.c_int32),
        ("eps", ctypes.c_float), ("clamp_delta", ctypes.c_float), ("state_dtype", ctypes.c_int32),
        ("impl", ctypes.c_int32), ("router", ctypes.c_int32), ("attn_aug", ctypes.c_int32),
    ]


def make_dims(T, N, k, m, C, Kr=1, S=None, kappa=(4, 8, 12), sinkhorn_iters=20, gram_schmidt=1,
              eps=1e-5, clamp_delta=1e-6, state="bf16", impl=XHC_IMPL_AUTO, router="sigmoid",
              attn_aug=0) -> Dims:
    d = Dims()
    d.T, d.S = T, (S if S else max(T, 1))
    d.N, d.k, d.m, d.C, d.Kr = N, k, m, C, Kr
    kap = list(kappa) + [0] * (3 - len(kappa))
    d.kappa = (ctypes.c_int32 * 3)(*kap[:3])
    d.sinkhorn_iters, d.gram_schmidt = sinkhorn_iters, gram_schmidt
    d.eps, d.clamp_delta = eps, clamp_delta
    d.state_dtype = XHC_BF16 if state == "bf16" else XHC_F32
    d.impl = impl
    d.router = XHC_ROUTER_SOFTMAX if router in ("softmax", XHC_ROUTER_SOFTMAX) else XHC_ROUTER_SIGMOID
    d.attn_aug = int(attn_aug)
    return d


def _int32(**values):
    """Refuses what a 32-bit field would cut to other values (ctypes does so without a word)."""
    for name, v in values.items():
        if not -2 ** 31 <= v < 2 ** 31:
            raise ValueError(f"{name} does not fit 32 bits: {v}")


class Heads(ctypes.Structure):
    _fields_ = [
        ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32), ("R", ctypes.c_int32),
        ("pairs", ctypes.c_int32), ("window", ctypes.c_int32), ("scale", ctypes.c_float), ("cap", ctypes.c_float),
    ]


def make_heads(Hq, Hkv, D, rotary=None, pairing="halves", window=0, scale=None, cap=0.0) -> Heads:
    """Heads of an attention-type sublayer: rotary is the number of channels that are rotated (all of a head's unless
    given), pairing "halves" or "neighbours", scale D^-1/2 unless given; window and cap 0 for none."""
    if pairing not in ("halves", "neighbours"):
        raise ValueError(f"pairing is 'halves' or 'neighbours', got {pairing!r}")
    rotary = D if rotary is None else rotary
    _int32(Hq=Hq, Hkv=Hkv, D=D, rotary=rotary, window=window)
    return Heads(Hq, Hkv, D, rotary, XHC_PAIRS_HALVES if pairing == "halves" else XHC_PAIRS_NEIGHBOURS, window,
                 D ** -0.5 if scale is None else scale, cap)


class Cache(ctypes.Structure):
    _fields_ = [("page", ctypes.c_int32), ("npages", ctypes.c_int32), ("B", ctypes.c_int32),
                ("per_seq", ctypes.c_int32)]


def dims_for(w, **kw) -> Dims:
    """Dims of a synth.Workload."""
    kw.setdefault("router", getattr(w, "router", "sigmoid"))
    kw.setdefault("gram_schmidt", getattr(w, "gram_schmidt", 1))
    kw.setdefault("attn_aug", getattr(w, "attn_aug", 0))
    return make_dims(w.T, w.N, w.k, w.m, w.C, Kr=w.Kr, S=w.S, kappa=w.kappa, state=w.state, **kw)


_lib = None
_P = ctypes.c_void_p
_D = ctypes.POINTER(Dims)
_H = ctypes.POINTER(Heads)
_C = ctypes.POINTER(Cache)
_SIGS = {
    "xhc_packed_full_bytes": (ctypes.c_size_t, [_D, ctypes.c_int32]),
    "xhc_packed_active_bytes": (ctypes.c_size_t, [_D, ctypes.c_int32, ctypes.c_int32]),
    "xhc_pack_full": (ctypes.c_int, [_D, ctypes.c_int32, _P, _P, _P, _P]),
    "xhc_pack_active": (ctypes.c_int, [_D, ctypes.c_int32, _P, _P, _P, _P]),
    "xhc_workspace_bytes": (ctypes.c_size_t, [_D, ctypes.c_int32, ctypes.c_int32]),
    "xhc_pre": (ctypes.c_int, [_D] + [_P] * 15 + [ctypes.c_size_t, _P]),
    "xhc_post": (ctypes.c_int, [_D] + [_P] * 9 + [ctypes.c_size_t, _P]),
    "xhc_saved_floats": (ctypes.c_size_t, [_D]),
    "xhc_post_noalloc": (ctypes.c_int, [_D] + [_P] * 9),
    "xhc_flash_pre": (ctypes.c_int, [_D, ctypes.c_int32] + [_P] * 16 + [ctypes.c_size_t, _P]),
    "xhc_flash_post": (ctypes.c_int, [_D, ctypes.c_int32, ctypes.c_int32] + [_P] * 19 + [ctypes.c_size_t, _P]),
    "xhc_flash_post_bwd": (ctypes.c_int, [_D, ctypes.c_int32, ctypes.c_int32] + [_P] * 30 + [ctypes.c_size_t, _P]),
    "xhc_flash_pre_bwd": (ctypes.c_int, [_D, ctypes.c_int32] + [_P] * 21 + [ctypes.c_size_t, _P]),
    "xhc_post_bwd": (ctypes.c_int, [_D] + [_P] * 16 + [ctypes.c_size_t, _P]),
    "xhc_pre_bwd": (ctypes.c_int, [_D] + [_P] * 27 + [ctypes.c_size_t, _P]),
    "xhc_stream_sum": (ctypes.c_int, [_D, _P, _P, _P]),
    "xhc_stream_sum_bwd": (ctypes.c_int, [_D, _P, _P, ctypes.c_int32, _P]),
    "xhc_pre_failures": (ctypes.c_int, [_P, _P, _P]),
    "xhc_rmsnorm_workspace_bytes": (ctypes.c_size_t, [_D]),
    "xhc_rmsnorm": (ctypes.c_int, [_D] + [_P] * 5),
    "xhc_rmsnorm_bwd": (ctypes.c_int, [_D] + [_P] * 7 + [ctypes.c_size_t, _P]),
    "xhc_packed_ffn_bytes": (ctypes.c_size_t, [_D, ctypes.c_int32, ctypes.c_int32]),
    "xhc_ffn_saved_bytes": (ctypes.c_size_t, [_D, ctypes.c_int32]),
    "xhc_ffn_workspace_bytes": (ctypes.c_size_t, [_D, ctypes.c_int32, ctypes.c_int32]),
    "xhc_pack_ffn": (ctypes.c_int, [_D, ctypes.c_int32, _P, _P, _P, ctypes.c_int32, _P, _P]),
    "xhc_ffn": (ctypes.c_int, [_D, ctypes.c_int32, ctypes.c_int32] + [_P] * 5 + [ctypes.c_size_t, _P]),
    "xhc_ffn_bwd": (ctypes.c_int, [_D, ctypes.c_int32, ctypes.c_int32] + [_P] * 9 + [ctypes.c_size_t, _P]),
    "xhc_rotate": (ctypes.c_int, [_D, _H] + [_P] * 3 + [ctypes.c_int64, ctypes.c_int32, _P, _P]),
    "xhc_attn_spans": (ctypes.c_int, [_D, _H, ctypes.c_int32] + [_P] * 4),
    "xhc_attn": (ctypes.c_int, [_D, _H] + [_P] * 6),
    "xhc_attn_saved_bytes": (ctypes.c_size_t, [_D, _H]),
    "xhc_attn_workspace_bytes": (ctypes.c_size_t, [_D, _H]),
    "xhc_attn_bwd": (ctypes.c_int, [_D, _H] + [_P] * 8 + [ctypes.c_size_t, _P]),
    "xhc_cache_bytes": (ctypes.c_size_t, [_H, _C]),
    "xhc_attn_cache_workspace_bytes": (ctypes.c_size_t, [_D, _H, _C]),
    "xhc_cache_append": (ctypes.c_int, [_D, _H, _C, _P, _P, ctypes.c_int64] + [_P] * 6),
    "xhc_cache_read": (ctypes.c_int, [_D, _H, _C] + [_P] * 7),
    "xhc_attn_cache": (ctypes.c_int, [_D, _H, _C] + [_P] * 8 + [ctypes.c_size_t, _P]),
    "xhc_grad_workspace_bytes": (ctypes.c_size_t, [ctypes.c_int32]),
    "xhc_grad_norm": (ctypes.c_int, [ctypes.c_int32] + [_P] * 5 + [ctypes.c_size_t, _P]),
    "xhc_grad_clip": (ctypes.c_int, [ctypes.c_int32] + [_P] * 3 + [ctypes.c_float] + [_P] * 3 + [ctypes.c_size_t, _P]),
    "xhc_status_string": (ctypes.c_char_p, [ctypes.c_int32]),
    "xhc_last_hip_error": (ctypes.c_char_p, []),
}


def lib():
    """Load libxhc.so once; raise if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2607_14530_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _lib = L
    return _lib


def declared_functions():
    """Names of the functions declared in include/xhc.h."""
    text = open(HEADER).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(xhc_[a-z0-9_]+)\s*\(", text)))


# ---------------------------------------------------------------- marshalling helpers

def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_cuda:
        raise ValueError("tensor arguments must be CUDA tensors")
    if not t.is_contiguous():
        raise ValueError("tensor arguments must be contiguous")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        dev = torch.cuda.current_device()
        try:                           # (not a documented name; current_stream makes an object first, 1.1 us)
            return torch._C._cuda_getCurrentRawStream(dev)
        except (AttributeError, TypeError):
            return torch.cuda.current_stream(dev).cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _call(name, *args):
    st = getattr(lib(), name)(*args)
    if st != XHC_OK:
        detail = f" ({lib().xhc_last_hip_error().decode()})" if st == XHC_EHIP else ""
        raise XhcError(name, st, detail)


def _expect(t, dtype, shape, name):
    if t.dtype != dtype or tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")


# ---------------------------------------------------------------- C entry points

def xhc_packed_full_bytes(d, npre):
    return lib().xhc_packed_full_bytes(ctypes.byref(d), npre)


def xhc_packed_active_bytes(d, Kq, with_res):
    return lib().xhc_packed_active_bytes(ctypes.byref(d), Kq, int(with_res))


def xhc_workspace_bytes(d, op, Q=0):
    return lib().xhc_workspace_bytes(ctypes.byref(d), op, Q)


def xhc_pack_full(d, npre, W_r, W_pre, packed, stream=None):
    _call("xhc_pack_full", ctypes.byref(d), npre, _ptr(W_r), _ptr(W_pre), _ptr(packed), _stream(stream))


def xhc_pack_active(d, Kq, W_post, W_res, packed, stream=None):
    _call("xhc_pack_active", ctypes.byref(d), Kq, _ptr(W_post), _ptr(W_res), _ptr(packed), _stream(stream))


def xhc_saved_floats(d):
    return lib().xhc_saved_floats(ctypes.byref(d))


def xhc_pre(d, X, packed_full, packed_act, alpha, b_pre, b_res, b_post, input, idx, p, Hpre, Hres, Hpost,
            saved, workspace, stream=None):
    _call("xhc_pre", ctypes.byref(d), _ptr(X), _ptr(packed_full), _ptr(packed_act), _ptr(alpha), _ptr(b_pre),
          _ptr(b_res), _ptr(b_post), _ptr(input), _ptr(idx), _ptr(p), _ptr(Hpre), _ptr(Hres), _ptr(Hpost),
          _ptr(saved), _ptr(workspace), workspace.numel() if workspace is not None else 0, _stream(stream))


def xhc_pre_failures(workspace, stream=None):
    """Waits for `stream`, then returns the number of bounded waits that gave
    up in the last xhc_pre call that used `workspace` (0 = none)."""
    n = ctypes.c_int32(0)
    _call("xhc_pre_failures", _ptr(workspace), ctypes.cast(ctypes.byref(n), ctypes.c_void_p), _stream(stream))
    return n.value


def xhc_post(d, X, F, conv_w, idx, p, Hres, Hpost, Xact_save, workspace, stream=None):
    _call("xhc_post", ctypes.byref(d), _ptr(X), _ptr(F), _ptr(conv_w), _ptr(idx), _ptr(p), _ptr(Hres),
          _ptr(Hpost), _ptr(Xact_save), _ptr(workspace), workspace.numel() if workspace is not None else 0,
          _stream(stream))


NOALLOC_SCRATCH_BYTES = 16 << 20   # XHC_NOALLOC_SCRATCH_BYTES


def xhc_post_noalloc(d, X, F, conv_w, idx, p, Hres, Hpost, Xact_save, stream=None):
    _call("xhc_post_noalloc", ctypes.byref(d), _ptr(X), _ptr(F), _ptr(conv_w), _ptr(idx), _ptr(p), _ptr(Hres),
          _ptr(Hpost), _ptr(Xact_save), _stream(stream))


def _nbytes(t):
    return t.numel() * t.element_size() if t is not None else 0


def xhc_flash_pre(d, Q, X, packed_full, packed_act1, alpha_pre, b_pre, alpha_post1, b_post1, input1, base, idx,
                  p, Hpre, Hpost1, saved, saved_act1, workspace, stream=None):
    _call("xhc_flash_pre", ctypes.byref(d), Q, _ptr(X), _ptr(packed_full), _ptr(packed_act1), _ptr(alpha_pre),
          _ptr(b_pre), _ptr(alpha_post1), _ptr(b_post1), _ptr(input1), _ptr(base), _ptr(idx), _ptr(p), _ptr(Hpre),
          _ptr(Hpost1), _ptr(saved), _ptr(saved_act1), _ptr(workspace), _nbytes(workspace), _stream(stream))


def xhc_flash_post(d, Q, q, X, F, conv_w, idx, p, Hpost, Hres, Hpre_next, base_next, input_next, packed_act_next,
                   alpha_next, b_post_next, b_res_next, Hpost_next, Hres_next, Xact_save, saved_next, workspace,
                   stream=None):
    _call("xhc_flash_post", ctypes.byref(d), Q, q, _ptr(X), _ptr(F), _ptr(conv_w), _ptr(idx), _ptr(p),
          _ptr(Hpost), _ptr(Hres), _ptr(Hpre_next), _ptr(base_next), _ptr(input_next), _ptr(packed_act_next),
          _ptr(alpha_next), _ptr(b_post_next), _ptr(b_res_next), _ptr(Hpost_next), _ptr(Hres_next),
          _ptr(Xact_save), _ptr(saved_next), _ptr(workspace), _nbytes(workspace), _stream(stream))


def xhc_flash_post_bwd(d, Q, q, dXn, da, Xact, F, conv_w, idx, p, Hpost, Hres, packed_act, W_post, W_res,
                       alpha_post, alpha_res, b_post, b_res, Hpre_q, d_input, saved_act, dF, dconv_w, dW_post,
                       dalpha_post, db_post, dW_res, dalpha_res, db_res, dp, dHpre_act, workspace, stream=None):
    _call("xhc_flash_post_bwd", ctypes.byref(d), Q, q, _ptr(dXn), _ptr(da), _ptr(Xact), _ptr(F), _ptr(conv_w),
          _ptr(idx), _ptr(p), _ptr(Hpost), _ptr(Hres), _ptr(packed_act), _ptr(W_post), _ptr(W_res),
          _ptr(alpha_post), _ptr(alpha_res), _ptr(b_post), _ptr(b_res), _ptr(Hpre_q), _ptr(d_input),
          _ptr(saved_act), _ptr(dF),
          _ptr(dconv_w), _ptr(dW_post), _ptr(dalpha_post), _ptr(db_post), _ptr(dW_res), _ptr(dalpha_res),
          _ptr(db_res), _ptr(dp), _ptr(dHpre_act), _ptr(workspace), _nbytes(workspace), _stream(stream))


def xhc_flash_pre_bwd(d, Q, X, packed_full, W_r, W_pre, alpha_pre, b_pre, idx, p, Hpre, saved, d_input, dHpre_act,
                      dp, dXn, da0, dX, dW_r, dW_pre, dalpha_pre, db_pre, workspace, stream=None):
    _call("xhc_flash_pre_bwd", ctypes.byref(d), Q, _ptr(X), _ptr(packed_full), _ptr(W_r), _ptr(W_pre),
          _ptr(alpha_pre), _ptr(b_pre), _ptr(idx), _ptr(p), _ptr(Hpre), _ptr(saved), _ptr(d_input),
          _ptr(dHpre_act), _ptr(dp),
          _ptr(dXn), _ptr(da0), _ptr(dX), _ptr(dW_r), _ptr(dW_pre), _ptr(dalpha_pre), _ptr(db_pre),
          _ptr(workspace), _nbytes(workspace), _stream(stream))


def xhc_post_bwd(d, dXn, X, Xact, F, conv_w, idx, p, Hres, Hpost, dX, dF, dHres, dHpost, dp, dconv_w, workspace,
                 stream=None):
    _call("xhc_post_bwd", ctypes.byref(d), _ptr(dXn), _ptr(X), _ptr(Xact), _ptr(F), _ptr(conv_w), _ptr(idx),
          _ptr(p), _ptr(Hres), _ptr(Hpost), _ptr(dX), _ptr(dF), _ptr(dHres), _ptr(dHpost), _ptr(dp), _ptr(dconv_w),
          _ptr(workspace), _nbytes(workspace), _stream(stream))


def xhc_pre_bwd(d, X, packed_full, W_r, W_pre, W_res, W_post, alpha, b_res, saved, idx, p, Hpre, Hpost, d_input,
                dHres, dHpost, dp, dX, dW_r, dW_pre, dW_res, dW_post, dalpha, db_pre, db_res, db_post, workspace,
                stream=None):
    _call("xhc_pre_bwd", ctypes.byref(d), _ptr(X), _ptr(packed_full), _ptr(W_r), _ptr(W_pre), _ptr(W_res),
          _ptr(W_post), _ptr(alpha), _ptr(b_res), _ptr(saved), _ptr(idx), _ptr(p), _ptr(Hpre), _ptr(Hpost),
          _ptr(d_input), _ptr(dHres), _ptr(dHpost), _ptr(dp), _ptr(dX), _ptr(dW_r), _ptr(dW_pre), _ptr(dW_res),
          _ptr(dW_post), _ptr(dalpha), _ptr(db_pre), _ptr(db_res), _ptr(db_post), _ptr(workspace),
          _nbytes(workspace), _stream(stream))


def xhc_stream_sum(d, X, out, stream=None):
    _call("xhc_stream_sum", ctypes.byref(d), _ptr(X), _ptr(out), _stream(stream))


def xhc_stream_sum_bwd(d, dout, dX, accumulate=False, stream=None):
    _call("xhc_stream_sum_bwd", ctypes.byref(d), _ptr(dout), _ptr(dX), int(bool(accumulate)), _stream(stream))


def xhc_rmsnorm_workspace_bytes(d):
    return lib().xhc_rmsnorm_workspace_bytes(ctypes.byref(d))


def xhc_rmsnorm(d, x, gain, y, rstd, stream=None):
    _call("xhc_rmsnorm", ctypes.byref(d), _ptr(x), _ptr(gain), _ptr(y), _ptr(rstd), _stream(stream))


def xhc_rmsnorm_bwd(d, x, gain, rstd, dy, dx, dgain, workspace, stream=None):
    _call("xhc_rmsnorm_bwd", ctypes.byref(d), _ptr(x), _ptr(gain), _ptr(rstd), _ptr(dy), _ptr(dx), _ptr(dgain),
          _ptr(workspace), _nbytes(workspace), _stream(stream))


def xhc_packed_ffn_bytes(d, H, with_bwd):
    return lib().xhc_packed_ffn_bytes(ctypes.byref(d), H, int(with_bwd))


def xhc_ffn_saved_bytes(d, H):
    return lib().xhc_ffn_saved_bytes(ctypes.byref(d), H)


def xhc_ffn_workspace_bytes(d, H, backward):
    return lib().xhc_ffn_workspace_bytes(ctypes.byref(d), H, int(backward))


def xhc_pack_ffn(d, H, W_gate, W_up, W_down, with_bwd, packed, stream=None):
    _call("xhc_pack_ffn", ctypes.byref(d), H, _ptr(W_gate), _ptr(W_up), _ptr(W_down), int(with_bwd), _ptr(packed),
          _stream(stream))


def xhc_ffn(d, H, act, input, packed, F, saved, workspace, stream=None):
    _call("xhc_ffn", ctypes.byref(d), H, act, _ptr(input), _ptr(packed), _ptr(F), _ptr(saved), _ptr(workspace),
          _nbytes(workspace), _stream(stream))


def xhc_ffn_bwd(d, H, act, input, packed, saved, dF, d_input, dW_gate, dW_up, dW_down, workspace, stream=None):
    _call("xhc_ffn_bwd", ctypes.byref(d), H, act, _ptr(input), _ptr(packed), _ptr(saved), _ptr(dF), _ptr(d_input),
          _ptr(dW_gate), _ptr(dW_up), _ptr(dW_down), _ptr(workspace), _nbytes(workspace), _stream(stream))


def xhc_rotate(d, h, in_, pos, table, positions, inverse, out, stream=None):
    _call("xhc_rotate", ctypes.byref(d), ctypes.byref(h), _ptr(in_), _ptr(pos), _ptr(table), positions,
          int(bool(inverse)), _ptr(out), _stream(stream))


def xhc_attn_spans(d, h, n, starts, prefix, span, stream=None):
    _call("xhc_attn_spans", ctypes.byref(d), ctypes.byref(h), n, _ptr(starts), _ptr(prefix), _ptr(span),
          _stream(stream))


def xhc_attn(d, h, qkv, span, slopes, out, saved, stream=None):
    _call("xhc_attn", ctypes.byref(d), ctypes.byref(h), _ptr(qkv), _ptr(span), _ptr(slopes), _ptr(out), _ptr(saved),
          _stream(stream))


def xhc_attn_saved_bytes(d, h):
    return lib().xhc_attn_saved_bytes(ctypes.byref(d), ctypes.byref(h))


def xhc_attn_workspace_bytes(d, h):
    return lib().xhc_attn_workspace_bytes(ctypes.byref(d), ctypes.byref(h))


def xhc_attn_bwd(d, h, qkv, span, slopes, out, saved, dout, dqkv, workspace, stream=None):
    _call("xhc_attn_bwd", ctypes.byref(d), ctypes.byref(h), _ptr(qkv), _ptr(span), _ptr(slopes), _ptr(out), _ptr(saved),
          _ptr(dout), _ptr(dqkv), _ptr(workspace), _nbytes(workspace), _stream(stream))


def xhc_cache_bytes(h, c):
    return lib().xhc_cache_bytes(ctypes.byref(h), ctypes.byref(c))


def xhc_attn_cache_workspace_bytes(d, h, c):
    return lib().xhc_attn_cache_workspace_bytes(ctypes.byref(d), ctypes.byref(h), ctypes.byref(c))


def xhc_cache_append(d, h, c, qkv, table, positions, starts, lens, pages, pool, q, stream=None):
    _call("xhc_cache_append", ctypes.byref(d), ctypes.byref(h), ctypes.byref(c), _ptr(qkv), _ptr(table), positions,
          _ptr(starts), _ptr(lens), _ptr(pages), _ptr(pool), _ptr(q), _stream(stream))


def xhc_cache_read(d, h, c, starts, lens, pages, pool, k, v, stream=None):
    _call("xhc_cache_read", ctypes.byref(d), ctypes.byref(h), ctypes.byref(c), _ptr(starts), _ptr(lens), _ptr(pages),
          _ptr(pool), _ptr(k), _ptr(v), _stream(stream))


def xhc_attn_cache(d, h, c, q, slopes, starts, lens, pages, pool, out, workspace, stream=None):
    _call("xhc_attn_cache", ctypes.byref(d), ctypes.byref(h), ctypes.byref(c), _ptr(q), _ptr(slopes), _ptr(starts),
          _ptr(lens), _ptr(pages), _ptr(pool), _ptr(out), _ptr(workspace), _nbytes(workspace), _stream(stream))


_GRAD_DTYPES = {torch.bfloat16: XHC_BF16, torch.float32: XHC_F32}


def _ptrs(tensors):
    """Host array of the tensors' addresses."""
    for t in tensors:
        if not (t.is_cuda and t.is_contiguous()):
            _ptr(t)
    return (_P * len(tensors))(*[t.data_ptr() for t in tensors])


def _grad_arrays(grads):
    """Host arrays of the tensors' addresses, counts and dtypes."""
    for g in grads:
        if g.dtype not in _GRAD_DTYPES:
            raise ValueError(f"gradients are bf16 or fp32, got {g.dtype}")
    n = len(grads)
    return (_ptrs(grads), (ctypes.c_int64 * n)(*[g.numel() for g in grads]),
            (ctypes.c_int32 * n)(*[_GRAD_DTYPES[g.dtype] for g in grads]))


def xhc_grad_workspace_bytes(n):
    return lib().xhc_grad_workspace_bytes(n)


def xhc_grad_norm(grads, norm, workspace, stream=None):
    ptrs, counts, dtypes = _grad_arrays(grads)
    _call("xhc_grad_norm", len(grads), ptrs, counts, dtypes, _ptr(norm), _ptr(workspace), _nbytes(workspace),
          _stream(stream))


def xhc_grad_clip(grads, max_norm, outs, norm, workspace, stream=None):
    """outs: a list of the gradients' shapes and dtypes (the gradients themselves for in place)."""
    ptrs, counts, dtypes = _grad_arrays(grads)
    to = ptrs
    if outs is not grads:
        if len(outs) != len(grads):
            raise ValueError(f"{len(grads)} gradients and {len(outs)} outputs")
        for g, o in zip(grads, outs):
            if o.dtype is not g.dtype or o.shape != g.shape:
                _expect(o, g.dtype, g.shape, "output of a gradient")
        to = _ptrs(outs)
    _call("xhc_grad_clip", len(grads), ptrs, counts, dtypes, max_norm, to, _ptr(norm), _ptr(workspace),
          _nbytes(workspace), _stream(stream))


# ---------------------------------------------------------------- convenience bundle

def _bytes(n, device):
    return torch.empty(max(int(n), 1), dtype=torch.uint8, device=device)


class Sublayer:
    """One full xHC sublayer: packed weights, parameters and output buffers.

    ``weights`` is a dict as produced by synth.sublayer_inputs (W_r, W_pre,
    W_res, W_post fp32; alpha [3]; b_pre, b_res, b_post; conv_w or None).
    """

    def __init__(self, d: Dims, weights, device="cuda"):
        self.d = d
        T, N, k, C, Kr = d.T, d.N, d.k, d.C, d.Kr
        dev = torch.device(device)
        g = {n: (v.to(dev).contiguous() if torch.is_tensor(v) else v) for n, v in weights.items()}
        self.packed_full = _bytes(xhc_packed_full_bytes(d, 1), dev)
        self.packed_act = _bytes(xhc_packed_active_bytes(d, Kr, 1), dev)
        xhc_pack_full(d, 1, g["W_r"], g["W_pre"], self.packed_full)
        xhc_pack_active(d, Kr, g["W_post"], g["W_res"], self.packed_act)
        self.alpha, self.b_pre, self.b_res, self.b_post = g["alpha"], g["b_pre"], g["b_res"], g["b_post"]
        self.conv_w = g.get("conv_w")
        sdt = torch.bfloat16 if d.state_dtype == XHC_BF16 else torch.float32
        self.input = torch.empty(T, C, dtype=sdt, device=dev)
        self.idx = torch.empty(T, k, dtype=torch.int32, device=dev)
        self.p = torch.empty(T, k, dtype=torch.float32, device=dev)
        self.Hpre = torch.empty(T, N, dtype=torch.float32, device=dev)
        self.Hres = torch.empty(T, k, k, dtype=torch.float32, device=dev)
        self.Hpost = torch.empty(T, k, Kr, dtype=torch.float32, device=dev)
        self.ws_pre = _bytes(xhc_workspace_bytes(d, XHC_OP_PRE), dev)
        self.ws_post = _bytes(xhc_workspace_bytes(d, XHC_OP_POST), dev)

    def pre(self, X, stream=None, saved=None):
        xhc_pre(self.d, X, self.packed_full, self.packed_act, self.alpha, self.b_pre, self.b_res, self.b_post,
                self.input, self.idx, self.p, self.Hpre, self.Hres, self.Hpost, saved, self.ws_pre, stream)
        return self.input

    def post(self, X, F, stream=None, Xact_save=None):
        xhc_post(self.d, X, F, self.conv_w, self.idx, self.p, self.Hres, self.Hpost, Xact_save, self.ws_post,
                 stream)
        return X

    def pre_failures(self, stream=None):
        """Bounded waits that gave up in the last pre() (waits for the stream)."""
        return xhc_pre_failures(self.ws_pre, stream)


def flash_Kq(d, q):
    """Write-back components of sublayer q (1-based) of a sharing group
    (attention-type sublayers have one unless d.attn_aug)."""
    return 1 if (q % 2 == 1 and not d.attn_aug) else d.Kr


class FlashGroup:
    """One xHC-Flash sharing group of Q sublayers: packed weights, parameters
    and output buffers.  ``weights`` is a dict as produced by
    synth.flash_inputs.  ``run(X, F_list)`` calls xhc_flash_pre and then
    xhc_flash_post for q = 1..Q; in a model the sublayer outputs F_q would be
    computed from ``inputs[q-1]`` between the calls (``step`` does one)."""

    def __init__(self, d: Dims, Q: int, weights, device="cuda"):
        assert Q in (2, 4)
        self.d, self.Q = d, Q
        T, N, k, C = d.T, d.N, d.k, d.C
        dev = torch.device(device)
        g = {n: v for n, v in weights.items()}
        f32 = dict(dtype=torch.float32, device=dev)
        self.packed_full = _bytes(xhc_packed_full_bytes(d, Q), dev)
        W_pre = torch.stack([w.to(dev) for w in g["W_pre_list"]]).contiguous()
        xhc_pack_full(d, Q, g["W_r"].to(dev).contiguous(), W_pre, self.packed_full)
        self.packed_act = []
        for q in range(1, Q + 1):
            Kq = flash_Kq(d, q)
            W_res = g["W_res"].to(dev).contiguous() if q == Q else None
            buf = _bytes(xhc_packed_active_bytes(d, Kq, W_res is not None), dev)
            xhc_pack_active(d, Kq, g["W_post_list"][q - 1].to(dev).contiguous(), W_res, buf)
            self.packed_act.append(buf)
        self.alpha_pre = torch.tensor(g["alpha_pre"], **f32)
        self.b_pre = torch.stack([b.to(dev) for b in g["b_pre"]]).contiguous().float()
        # alpha_next[q-1] = (alpha_post of sublayer q, alpha_res)
        self.alpha_post = [torch.tensor([g["alpha_post"][q], g["alpha_res"]], **f32) for q in range(Q)]
        self.b_post = [b.to(dev).contiguous().float() for b in g["b_post"]]
        self.b_res = g["b_res"].to(dev).contiguous().float()
        self.conv_w = [(c.to(dev).contiguous() if c is not None else None) for c in g["conv_w_list"]]
        sdt = torch.bfloat16 if d.state_dtype == XHC_BF16 else torch.float32
        self.inputs = [torch.empty(T, C, dtype=sdt, device=dev) for _ in range(Q)]
        self.base = torch.empty(Q - 1, T, C, dtype=sdt, device=dev)
        self.idx = torch.empty(T, k, dtype=torch.int32, device=dev)
        self.p = torch.empty(T, k, **f32)
        self.Hpre = torch.empty(Q, T, N, **f32)
        self.Hpost = [torch.empty(T, k, flash_Kq(d, q), **f32) for q in range(1, Q + 1)]
        self.Hres = torch.empty(T, k, k, **f32)
        self.ws_pre = _bytes(xhc_workspace_bytes(d, XHC_OP_FLASH_PRE, Q), dev)
        self.ws_post = _bytes(xhc_workspace_bytes(d, XHC_OP_FLASH_POST, Q), dev)

    def pre(self, X, stream=None, saved=None, saved_act1=None):
        xhc_flash_pre(self.d, self.Q, X, self.packed_full, self.packed_act[0], self.alpha_pre, self.b_pre,
                      self.alpha_post[0], self.b_post[0], self.inputs[0], self.base, self.idx, self.p, self.Hpre,
                      self.Hpost[0], saved, saved_act1, self.ws_pre, stream)

    def step(self, q, X, F, stream=None, Xact_save=None, saved_next=None):
        """Write-back of sublayer q (1-based); for q < Q also forms inputs[q]."""
        Q = self.Q
        last = q == Q
        nxt = None if last else q          # 0-based index of sublayer q + 1
        xhc_flash_post(
            self.d, Q, q, X, F, self.conv_w[q - 1], self.idx, self.p, self.Hpost[q - 1],
            self.Hres if last else None,
            None if last else self.Hpre[nxt], None if last else self.base[nxt - 1],
            None if last else self.inputs[nxt], None if last else self.packed_act[nxt],
            None if last else self.alpha_post[nxt], None if last else self.b_post[nxt],
            self.b_res if (not last and q + 1 == Q) else None,
            None if last else self.Hpost[nxt], self.Hres if (not last and q + 1 == Q) else None,
            Xact_save, saved_next, self.ws_post, stream)

    def run(self, X, F_list, stream=None):
        self.pre(X, stream)
        for q in range(1, self.Q + 1):
            self.step(q, X, F_list[q - 1], stream)
        return X


class TrainableFlashGroup(FlashGroup):
    """A FlashGroup that keeps what the backward needs and runs it.

    forward(X, F_list): xhc_flash_pre, then xhc_flash_post for q = 1..Q saving
    the active rows before each write-back; X is updated in place.
    backward(X0, dXn, d_inputs, F_list): the reverse sweep, xhc_flash_post_bwd
    for q = Q..1 then xhc_flash_pre_bwd on the group-entry state X0 (the
    caller keeps X0: the group overwrites the active rows of X).  Returns a
    dict of gradients keyed like the oracle's (X, F_list, conv_w_list, W_r,
    W_pre_list, W_post_list, W_res, alpha_pre, b_pre, alpha_post, b_post,
    alpha_res, b_res)."""

    def __init__(self, d: Dims, Q: int, weights, device="cuda"):
        super().__init__(d, Q, weights, device)
        dev = torch.device(device)
        T, N, k, C = d.T, d.N, d.k, d.C
        f32 = dict(dtype=torch.float32, device=dev)
        self.W_r = weights["W_r"].to(dev).contiguous().float()
        self.W_pre = torch.stack([w.to(dev) for w in weights["W_pre_list"]]).contiguous().float()
        self.W_post = [w.to(dev).contiguous().float() for w in weights["W_post_list"]]
        self.W_res = weights["W_res"].to(dev).contiguous().float()
        self.a_post = [torch.tensor([a], **f32) for a in weights["alpha_post"]]
        self.a_res = torch.tensor([weights["alpha_res"]], **f32)
        self.Xact = [torch.empty(T, k, C, dtype=self.inputs[0].dtype, device=dev) for _ in range(Q)]
        # the routing records of the group entry, one per pre-map (xhc_flash_pre writes them)
        self.saved = torch.empty(Q, T, 2 * N + k + k * k + 4, **f32)
        # each sublayer's mapping record (its logits and RMS statistic; xhc_flash_pre
        # writes sublayer 1's, xhc_flash_post q the one of q + 1)
        self.saved_act = [torch.empty(T, 2 * k + k * flash_Kq(d, q) + k * k + 4, **f32) for q in range(1, Q + 1)]
        self.ws_post_bwd = _bytes(xhc_workspace_bytes(d, XHC_OP_FLASH_POST_BWD, Q), dev)
        self.ws_pre_bwd = _bytes(xhc_workspace_bytes(d, XHC_OP_FLASH_PRE_BWD, Q), dev)

    def forward(self, X, F_list, stream=None):
        self.pre(X, stream, saved=self.saved, saved_act1=self.saved_act[0])
        for q in range(1, self.Q + 1):
            self.step(q, X, F_list[q - 1], stream, Xact_save=self.Xact[q - 1],
                      saved_next=self.saved_act[q] if q < self.Q else None)
        return X

    def backward(self, X0, dXn, d_inputs, F_list, stream=None, in_place=False, recompute=False):
        """Group reverse given dL/dX' (dXn) and dL/d input_q (d_inputs: a list
        of Q [T, C] tensors, or one [Q, T, C] tensor).  With in_place, dL/dX
        is formed in dXn itself (only the active rows of each token are
        rewritten before the pre-map passes add to it) and g["X"] is dXn.
        The entry reverse reads the routing records the forward saved, or,
        with recompute, forms them again from X0."""
        d, Q = self.d, self.Q
        T, N, k, C = d.T, d.N, d.k, d.C
        dev = X0.device
        f32 = dict(dtype=torch.float32, device=dev)
        sdt = self.inputs[0].dtype
        g = {"F_list": [None] * Q, "conv_w_list": [None] * Q, "W_post_list": [None] * Q, "b_post": [None] * Q}
        da = torch.empty(T, k, C, **f32)
        dp = torch.zeros(T, k, **f32)
        dhact = torch.empty(max(Q - 1, 1), T, k, **f32)
        a_post = torch.empty(Q, **f32)
        g["W_res"], g["b_res"] = torch.empty_like(self.W_res), torch.empty(k * k, **f32)
        a_res = torch.empty(1, **f32)
        for q in range(Q, 0, -1):
            last, Kq = q == Q, flash_Kq(d, q)
            g["F_list"][q - 1] = torch.empty(T, C, dtype=sdt, device=dev)
            g["conv_w_list"][q - 1] = torch.empty_like(self.conv_w[q - 1]) if self.conv_w[q - 1] is not None else None
            g["W_post_list"][q - 1] = torch.empty_like(self.W_post[q - 1])
            g["b_post"][q - 1] = torch.empty(k * Kq, **f32)
            xhc_flash_post_bwd(
                d, Q, q, dXn if last else None, da, self.Xact[q - 1], F_list[q - 1], self.conv_w[q - 1], self.idx,
                self.p, self.Hpost[q - 1], self.Hres if last else None, self.packed_act[q - 1], self.W_post[q - 1],
                self.W_res if last else None, self.a_post[q - 1], self.a_res if last else None, self.b_post[q - 1],
                self.b_res if last else None, self.Hpre[q - 1] if q >= 2 else None,
                d_inputs[q - 1] if q >= 2 else None, None if recompute else self.saved_act[q - 1],
                g["F_list"][q - 1], g["conv_w_list"][q - 1],
                g["W_post_list"][q - 1], a_post[q - 1:q], g["b_post"][q - 1], g["W_res"] if last else None,
                a_res if last else None, g["b_res"] if last else None, dp, dhact[q - 2] if q >= 2 else None,
                self.ws_post_bwd, stream)
        din = d_inputs.contiguous() if torch.is_tensor(d_inputs) else torch.stack(list(d_inputs)).contiguous()
        g["X"] = dXn if in_place else torch.empty_like(X0)
        g["W_r"], g["W_pre"] = torch.empty_like(self.W_r), torch.empty_like(self.W_pre)
        g["alpha_pre"], g["b_pre"] = torch.empty(Q, **f32), torch.empty(Q, N, **f32)
        xhc_flash_pre_bwd(d, Q, X0, self.packed_full, self.W_r, self.W_pre, self.alpha_pre, self.b_pre, self.idx,
                          self.p, self.Hpre, None if recompute else self.saved, din, dhact, dp, dXn, da, g["X"],
                          g["W_r"], g["W_pre"],
                          g["alpha_pre"], g["b_pre"], self.ws_pre_bwd, stream)
        g["W_pre_list"] = list(g.pop("W_pre"))
        g["b_pre"] = list(g["b_pre"])
        g["alpha_post"], g["alpha_res"] = a_post, a_res[0]
        return g


class TrainableSublayer(Sublayer):
    """A Sublayer that keeps what the backward needs and runs it.

    forward(X, F): xhc_pre (saving the per-token logits / statistics) and
    xhc_post (saving the pre-update active rows); X is updated in place.
    backward(X, dXn, d_input, F): xhc_post_bwd (restores X to the pre-update
    state) then xhc_pre_bwd; returns a dict of gradients."""

    def __init__(self, d: Dims, weights, device="cuda"):
        super().__init__(d, weights, device)
        dev = torch.device(device)
        self.W = {n: weights[n].to(dev).contiguous().float() for n in ("W_r", "W_pre", "W_res", "W_post")}
        T, N, k, C, Kr = d.T, d.N, d.k, d.C, d.Kr
        sdt = self.input.dtype
        self.saved = torch.empty(T, xhc_saved_floats(d), dtype=torch.float32, device=dev)
        self.Xact = torch.empty(T, k, C, dtype=sdt, device=dev)
        self.ws_post_bwd = _bytes(xhc_workspace_bytes(d, XHC_OP_POST_BWD), dev)
        self.ws_pre_bwd = _bytes(xhc_workspace_bytes(d, XHC_OP_PRE_BWD), dev)

    def forward(self, X, F, stream=None):
        self.pre(X, stream, saved=self.saved)
        self.post(X, F, stream, Xact_save=self.Xact)
        return X

    def backward(self, X, dXn, d_input, F, stream=None, in_place=False):
        g = self.backward_post(X, dXn, F, stream, in_place)
        return self.backward_pre(X, d_input, g, stream)

    def backward_post(self, X, dXn, F, stream=None, in_place=False):
        """xhc_post_bwd: restores X to the state xhc_pre saw and returns the
        partial gradients, dL/dF among them (for the sublayer's own backward).
        With in_place, dL/dX is formed in dXn itself (only the k active rows
        of each token are rewritten) and g["X"] is dXn."""
        d = self.d
        T, N, k, C, Kr = d.T, d.N, d.k, d.C, d.Kr
        dev = X.device
        f32 = dict(dtype=torch.float32, device=dev)
        g = {"X": dXn if in_place else torch.empty_like(X), "F": torch.empty_like(F),
             "dHres": torch.empty(T, k, k, **f32),
             "dHpost": torch.empty(T, k, Kr, **f32), "dp": torch.empty(T, k, **f32),
             "conv_w": torch.empty_like(self.conv_w) if self.conv_w is not None else None}
        xhc_post_bwd(d, dXn, X, self.Xact, F, self.conv_w, self.idx, self.p, self.Hres, self.Hpost, g["X"], g["F"],
                     g["dHres"], g["dHpost"], g["dp"], g["conv_w"], self.ws_post_bwd, stream)
        return g

    def backward_pre(self, X, d_input, g, stream=None):
        """xhc_pre_bwd given dL/d input: completes g (g["X"] becomes the full dL/dX)."""
        d = self.d
        N, k, Kr = d.N, d.k, d.Kr
        f32 = dict(dtype=torch.float32, device=X.device)
        for n in ("W_r", "W_pre", "W_res", "W_post"):
            g[n] = torch.empty_like(self.W[n])
        g["alpha"] = torch.empty(3, **f32)
        g["b_pre"], g["b_res"], g["b_post"] = (torch.empty(N, **f32), torch.empty(k * k, **f32),
                                               torch.empty(k * Kr, **f32))
        xhc_pre_bwd(d, X, self.packed_full, self.W["W_r"], self.W["W_pre"], self.W["W_res"], self.W["W_post"],
                    self.alpha, self.b_res, self.saved, self.idx, self.p, self.Hpre, self.Hpost, d_input,
                    g["dHres"], g["dHpost"], g["dp"], g["X"], g["W_r"], g["W_pre"], g["W_res"], g["W_post"],
                    g["alpha"], g["b_pre"], g["b_res"], g["b_post"], self.ws_pre_bwd, stream)
        return g


class Stack:
    """L xHC sublayers chained on one in-place state buffer, then the final
    stream reduction (App. "Final Stream Reduction").  Host-side sequencing of
    the C entry points only.

    ``layers`` is a list of TrainableSublayer.  forward(X, fns) runs, for each
    layer l, xhc_pre, F_l = fns[l](input_l) (the caller's attention / MLP
    function of the bf16 input) and xhc_post, keeping the F_l and the saved
    rows; it returns the reduced [T, C] output.  backward(X, d_out, fn_bwds)
    sweeps the layers in reverse: xhc_post_bwd restores layer l's pre-update
    state from its saved active rows, fn_bwds[l](dF_l) gives dL/d input_l for
    xhc_pre_bwd, and dL/dX flows to layer l - 1.  It returns the per-layer
    gradient dicts (last layer last) and dL/dX of the entry state; X is back
    at the entry state afterwards.
    """

    def __init__(self, layers):
        self.layers = list(layers)
        d0 = self.layers[0].d
        for sub in self.layers:
            if (sub.d.T, sub.d.N, sub.d.C, sub.d.state_dtype) != (d0.T, d0.N, d0.C, d0.state_dtype):
                raise ValueError("layers of a stack share T, N, C and the state dtype")
        self.F = [None] * len(self.layers)

    def forward(self, X, fns, stream=None):
        for l, sub in enumerate(self.layers):
            sub.pre(X, stream, saved=sub.saved)
            F = fns[l](sub.input)
            self.F[l] = F
            sub.post(X, F, stream, Xact_save=sub.Xact)
        d0 = self.layers[0].d
        out = torch.empty(d0.T, d0.C, dtype=X.dtype, device=X.device)
        xhc_stream_sum(d0, X, out, stream)
        return out

    def backward(self, X, d_out, fn_bwds, stream=None, in_place=True):
        """With in_place (default) the state gradient runs through one buffer
        (each xhc_post_bwd rewrites only the active rows): every layer's
        grads[l]["X"] is that buffer, holding dL/dX of the entry state at the
        end.  in_place=False keeps each layer's dL/dX in its own tensor."""
        d0 = self.layers[0].d
        dX = torch.empty_like(X)
        xhc_stream_sum_bwd(d0, d_out, dX, False, stream)
        grads = [None] * len(self.layers)
        for l in range(len(self.layers) - 1, -1, -1):
            sub = self.layers[l]
            g = sub.backward_post(X, dX, self.F[l], stream, in_place=in_place)
            d_input = fn_bwds[l](g["F"])
            g = sub.backward_pre(X, d_input, g, stream)
            grads[l] = g
            dX = g["X"]
        return grads, dX


# ---------------------------------------------------------------- the sublayer's own function

def _enqueues(dev):
    """Refuses a call of a bundle while another device is current: it would be enqueued there."""
    if dev.type == "cuda" and torch.cuda.current_device() != dev.index:
        raise ValueError(f"the current device is cuda:{torch.cuda.current_device()}, not the bundle's {dev}")


def _on(t, dev, name):
    """An argument of a bundle's call, on the bundle's device, which is the current one."""
    if t.device != dev:
        raise ValueError(f"{name} is on {t.device}, expected {dev}")
    _enqueues(dev)


def _here(device):
    """The device of a bundle: the current one, where its calls enqueue."""
    dev = torch.device(device)
    cur = torch.device("cuda", torch.cuda.current_device())
    if dev.type != "cuda" or (dev.index is not None and dev != cur):
        raise ValueError(f"{dev} is not the current device {cur}")
    return cur


def _within(stream):
    """The context in which temporaries of work on `stream` are made: their
    memory then belongs to that stream."""
    if stream is None:
        return contextlib.nullcontext()
    return torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream)))


def _state_dtype(d):
    return torch.bfloat16 if d.state_dtype == XHC_BF16 else torch.float32


class RMSNorm:
    """RMS norm of [T, C] rows with a gain (fp32 [C]); eps is d.eps.  The gain
    is read at every call: where it is contiguous on the device already it is
    not copied, and new values written to it count.  Outputs go to a buffer of
    this object, overwritten by its next forward."""

    def __init__(self, d: Dims, gain, device="cuda"):
        self.d, self.device = d, _here(device)
        _expect(gain, torch.float32, (d.C,), "gain")
        self.gain = gain.to(self.device).contiguous()
        self.y = torch.empty(d.T, d.C, dtype=_state_dtype(d), device=self.device)
        self.rstd = None

    def forward(self, x, stream=None):
        _expect(x, self.y.dtype, self.y.shape, "x")
        _on(x, self.device, "x")
        xhc_rmsnorm(self.d, x, self.gain, self.y, self.rstd, stream)
        return self.y


class TrainableRMSNorm(RMSNorm):
    """An RMSNorm that keeps what the backward needs and runs it: backward(dy)
    returns dL/dx of the last forward's x (read again: it must still hold its
    values) and leaves dL/dgain in grads["gain"]."""

    def __init__(self, d: Dims, gain, device="cuda"):
        super().__init__(d, gain, device)
        self.rstd = torch.empty(d.T, dtype=torch.float32, device=self.device)
        self.dx = torch.empty_like(self.y)
        self.grads = {"gain": torch.empty_like(self.gain)}
        self.ws = _bytes(xhc_rmsnorm_workspace_bytes(d), self.device)
        self.x = None

    def forward(self, x, stream=None):
        out = super().forward(x, stream)
        self.x = x                     # (of a forward that ran: a refused one changes nothing)
        return out

    def backward(self, dy, stream=None):
        if self.x is None:
            raise ValueError("backward without a forward")
        _expect(dy, self.y.dtype, self.y.shape, "dy")
        _on(dy, self.device, "dy")
        xhc_rmsnorm_bwd(self.d, self.x, self.gain, self.rstd, dy, self.dx, self.grads["gain"], self.ws, stream)
        return self.dx


class FeedForward:
    """Gated feed-forward block F = (act(x W_gate) * (x W_up)) W_down of [T, C]
    rows: packed weights and buffers.  ``weights`` holds W_gate, W_up [C, H]
    and W_down [H, C], fp32; act is "silu" or "gelu".  pack(weights) takes new
    values of them.  Outputs go to a buffer of this object, overwritten by its
    next forward."""

    with_bwd = 0

    def __init__(self, d: Dims, H: int, weights, act="silu", device="cuda"):
        if act not in ("silu", "gelu"):
            raise ValueError(f"act is 'silu' or 'gelu', got {act!r}")
        self.d, self.H, self.device = d, H, _here(device)
        self.act = XHC_ACT_SILU if act == "silu" else XHC_ACT_GELU
        self.F = torch.empty(d.T, d.C, dtype=_state_dtype(d), device=self.device)
        self.packed = _bytes(xhc_packed_ffn_bytes(d, H, self.with_bwd), self.device)
        self.ws = _bytes(xhc_ffn_workspace_bytes(d, H, 0), self.device)
        self.saved = None
        self.pack(weights)

    def pack(self, weights, stream=None):
        w = [weights[n] for n in ("W_gate", "W_up", "W_down")]
        for t, n in zip(w, ("W_gate", "W_up", "W_down")):
            _expect(t, torch.float32, (self.H, self.d.C) if n == "W_down" else (self.d.C, self.H), n)
        _enqueues(self.device)
        with _within(stream):
            w = [t.to(self.device).contiguous() for t in w]
        xhc_pack_ffn(self.d, self.H, *w, self.with_bwd, self.packed, stream)

    def forward(self, x, stream=None):
        _expect(x, self.F.dtype, self.F.shape, "x")
        _on(x, self.device, "x")
        xhc_ffn(self.d, self.H, self.act, x, self.packed, self.F, self.saved, self.ws, stream)
        return self.F


class TrainableFeedForward(FeedForward):
    """A FeedForward that keeps what the backward needs and runs it:
    backward(dF) returns dL/dx of the last forward's x (read again: it must
    still hold its values, as the input buffer of a sublayer does) and leaves
    dL/dW_gate, dL/dW_up and dL/dW_down in grads, in the state dtype."""

    with_bwd = 1

    def __init__(self, d: Dims, H: int, weights, act="silu", device="cuda"):
        super().__init__(d, H, weights, act, device)
        self.saved = _bytes(xhc_ffn_saved_bytes(d, H), self.device)
        self.ws_bwd = _bytes(xhc_ffn_workspace_bytes(d, H, 1), self.device)
        self.d_input = torch.empty_like(self.F)
        self.grads = {n: torch.empty((H, d.C) if n == "W_down" else (d.C, H), dtype=self.F.dtype, device=self.device)
                      for n in ("W_gate", "W_up", "W_down")}
        self.x = None

    def forward(self, x, stream=None):
        out = super().forward(x, stream)
        self.x = x                     # (of a forward that ran: a refused one changes nothing)
        return out

    def backward(self, dF, stream=None):
        if self.x is None:
            raise ValueError("backward without a forward")
        _expect(dF, self.F.dtype, self.F.shape, "dF")
        _on(dF, self.device, "dF")
        g = self.grads
        xhc_ffn_bwd(self.d, self.H, self.act, self.x, self.packed, self.saved, dF, self.d_input, g["W_gate"],
                    g["W_up"], g["W_down"], self.ws_bwd, stream)
        return self.d_input


def rotation_table(positions, R, base=10000.0, device="cuda"):
    """Cosines and sines [positions, R / 2, 2] of the angles p base^(-2 i / R), formed in 64 bits (the angles of far
    positions need them) and rounded to fp32.  A table of other frequencies is as good."""
    f = base ** (-2.0 * torch.arange(R // 2, dtype=torch.float64, device=device) / max(R, 1))
    a = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * f
    return torch.stack([torch.cos(a), torch.sin(a)], -1).float()


def _settle():
    """Waits for what a bundle's constructor has enqueued, and for earlier work in memory that it was given: its first
    call may then go to any stream.  (Where the constructor itself is captured there is nothing to wait for before the
    replay.)"""
    if not torch.cuda.is_current_stream_capturing():
        torch.cuda.current_stream().synchronize()


def _laid_out(t, device):
    """The tensor itself where it is contiguous on the device, else a copy that is."""
    c = t.to(device).contiguous()
    if c is not t:
        _settle()
    return c


def _table(h, table, device):
    if h.R == 0:
        return None, 0
    _expect(table, torch.float32, (table.shape[0], h.R // 2, 2), "table")
    return _laid_out(table, device), table.shape[0]


def _slopes(h, slopes, device):
    if slopes is None:
        return None
    _expect(slopes, torch.float32, (h.Hq,), "slopes")
    return _laid_out(slopes, device)


def _take(t, dtype, shape, dev, name):
    """The address of an argument of a call: of this dtype, shape (a tuple) and device."""
    if t.dtype is not dtype or t.shape != shape:
        _expect(t, dtype, shape, name)
    if t.get_device() != dev.index:
        raise ValueError(f"{name} is on {t.device}, expected {dev}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _version(t):
    """How often torch has changed t in place; None where it does not count."""
    return None if t.is_inference() else t._version


class Rotation:
    """Position rotation of the query and key heads of qkv [T, Hq + 2 Hkv, D] by a table of cosines and sines
    (rotation_table).  Positions are t % d.S unless given (pos [T] int32).  Forward and backward each have a buffer
    of this object for their output, overwritten by their next call; with ``out``, which may be the input itself, it
    goes there."""

    def __init__(self, d: Dims, h: Heads, table, device="cuda"):
        self.d, self.h, self.device = d, h, _here(device)
        self.table, self.positions = _table(h, table, self.device)
        self.shape, self.dtype = (d.T, h.Hq + 2 * h.Hkv, h.D), _state_dtype(d)
        self.buffers = [None, None]    # of forward, of backward

    def _run(self, x, pos, out, inverse, stream):
        at = _take(x, self.dtype, self.shape, self.device, "the heads")
        if pos is not None:
            pos = _take(pos, torch.int32, (self.d.T,), self.device, "pos")
        _enqueues(self.device)
        if out is None:
            if self.buffers[inverse] is None:
                with _within(stream):
                    self.buffers[inverse] = torch.empty(self.shape, dtype=self.dtype, device=self.device)
            out = self.buffers[inverse]
        else:
            _take(out, self.dtype, self.shape, self.device, "out")
        xhc_rotate(self.d, self.h, at, pos, self.table, self.positions, inverse, out, stream)
        return out

    def forward(self, qkv, pos=None, out=None, stream=None):
        return self._run(qkv, pos, out, 0, stream)

    def backward(self, dqkv, pos=None, out=None, stream=None):
        """The gradient of forward's input, given that of its output."""
        return self._run(dqkv, pos, out, 1, stream)


class Attention:
    """Attention of qkv [T, Hq + 2 Hkv, D]: forward(qkv, span) returns [T, Hq, D].  Without a span a token sees the
    tokens of its sequence (d.S) up to itself; spans() gives those of packed documents, also with prefixes that see
    themselves both ways.  slopes [Hq] fp32: of a bias -slope |i - j|.  Outputs go to buffers of this object,
    overwritten by its next call."""

    def __init__(self, d: Dims, h: Heads, slopes=None, device="cuda"):
        self.d, self.h, self.device = d, h, _here(device)
        self.slopes = _slopes(h, slopes, self.device)
        self.out = torch.empty(d.T, h.Hq, h.D, dtype=_state_dtype(d), device=self.device)
        self.shape = (d.T, h.Hq + 2 * h.Hkv, h.D)
        self.saved = None
        self.span = None
        _settle()

    def spans(self, starts=None, prefix=None, stream=None):
        """span [T, 2] of documents: document i has the tokens starts[i] .. starts[i + 1] - 1 (int32 [n + 1]), its
        first prefix[i] (int32 [n]) seen by all of it, as far as a window reaches back; without starts, of
        sequences."""
        n = 0 if starts is None else starts.numel() - 1
        if starts is not None:
            if n < 0:
                raise ValueError("starts holds one entry more than there are documents")
            _int32(documents=n)
            starts = _take(starts, torch.int32, (n + 1,), self.device, "starts")
        if prefix is not None:
            prefix = _take(prefix, torch.int32, (n,), self.device, "prefix")
        _enqueues(self.device)
        if self.span is None:
            with _within(stream):
                self.span = torch.empty(self.d.T, 2, dtype=torch.int32, device=self.device)
        xhc_attn_spans(self.d, self.h, n, starts, prefix, self.span, stream)
        return self.span

    def forward(self, qkv, span=None, stream=None):
        qkv = _take(qkv, self.out.dtype, self.shape, self.device, "qkv")
        if span is not None:
            span = _take(span, torch.int32, (self.d.T, 2), self.device, "span")
        _enqueues(self.device)
        xhc_attn(self.d, self.h, qkv, span, self.slopes, self.out, self.saved, stream)
        return self.out


class TrainableAttention(Attention):
    """An Attention that keeps what the backward needs and runs it: backward(dout) returns dL/dqkv of the last
    forward's qkv and span.  It reads them again, and the output that forward returned: they must still hold their
    values.  An output that torch has changed in place since then is refused."""

    def __init__(self, d: Dims, h: Heads, slopes=None, device="cuda"):
        super().__init__(d, h, slopes, device)
        self.saved = _bytes(xhc_attn_saved_bytes(d, h), self.device)
        self.dqkv = torch.empty(self.shape, dtype=self.out.dtype, device=self.device)
        self.ws = _bytes(xhc_attn_workspace_bytes(d, h), self.device)
        self.seen = None
        _settle()

    def forward(self, qkv, span=None, stream=None):
        out = super().forward(qkv, span, stream)
        self.seen = (qkv, span, _version(out))       # (of a forward that ran: a refused one changes nothing)
        return out

    def backward(self, dout, stream=None):
        if self.seen is None:
            raise ValueError("backward without a forward")
        qkv, span, version = self.seen
        if _version(self.out) != version:
            raise ValueError("the forward's output was changed in place: backward reads it again")
        dout = _take(dout, self.out.dtype, self.out.shape, self.device, "dout")
        _enqueues(self.device)
        xhc_attn_bwd(self.d, self.h, qkv, span, self.slopes, self.out, self.saved, dout, self.dqkv, self.ws, stream)
        return self.dqkv


class KVCache:
    """Paged cache of a layer's keys and values in 4 bits, for calls of d.T tokens.  ``sequences`` rows of a page table
    of ``per_sequence`` entries name pages of a pool of ``npages``, ``page`` tokens each; an entry that is no page
    (-1) is one that is not there.  Each call takes starts [sequences + 1], lens [sequences] and pages [sequences,
    per_sequence], int32 on the device: sequence b's newest tokens are starts[b] .. starts[b + 1] - 1 of the call's,
    the last of its lens[b].  ``pool``: that of another KVCache with the same heads, page and npages, for calls of
    another number of tokens.  Outputs go to buffers of this object, overwritten by its next call but for the rows of
    tokens that no sequence has or that lie outside its row of the page table (as in a padded batch), and in read() of
    tokens that are not stored: those keep what an earlier call left there, zeros at first."""

    def __init__(self, d: Dims, h: Heads, table, sequences, per_sequence, page=64, npages=None, slopes=None,
                 pool=None, device="cuda"):
        self.d, self.h, self.device = d, h, _here(device)
        npages = sequences * per_sequence if npages is None else npages
        _int32(page=page, npages=npages, sequences=sequences, per_sequence=per_sequence)
        self.c = Cache(page, npages, sequences, per_sequence)
        self.table, self.positions = _table(h, table, self.device)
        self.slopes = _slopes(h, slopes, self.device)
        n = xhc_cache_bytes(h, self.c)
        if n == 0:
            raise ValueError("a cache of these sizes is not supported")
        if pool is None:
            pool = torch.zeros(n, dtype=torch.uint8, device=self.device)
        _expect(pool, torch.uint8, (n,), "pool")
        _on(pool, self.device, "pool")
        self.pool = pool
        sdt = _state_dtype(d)
        # (k and v now and not by the first read: in a captured one the zeros would be part of every replay)
        self.q, self.out = (torch.zeros(d.T, h.Hq, h.D, dtype=sdt, device=self.device) for _ in range(2))
        self.k, self.v = (torch.zeros(d.T, h.Hkv, h.D, dtype=sdt, device=self.device) for _ in range(2))
        self.shape = (d.T, h.Hq + 2 * h.Hkv, h.D)
        self.ws = _bytes(xhc_attn_cache_workspace_bytes(d, h, self.c), self.device)
        _settle()

    def _check(self, starts, lens, pages):
        B = self.c.B
        at = (_take(starts, torch.int32, (B + 1,), self.device, "starts"),
              _take(lens, torch.int32, (B,), self.device, "lens"),
              _take(pages, torch.int32, (B, self.c.per_seq), self.device, "pages"))
        _enqueues(self.device)
        return at

    def append(self, qkv, starts, lens, pages, stream=None):
        """Stores the rotated key heads and the value heads of qkv [T, Hq + 2 Hkv, D]; returns the rotated query heads
        [T, Hq, D]."""
        qkv = _take(qkv, self.q.dtype, self.shape, self.device, "qkv")
        xhc_cache_append(self.d, self.h, self.c, qkv, self.table, self.positions,
                         *self._check(starts, lens, pages), self.pool, self.q, stream)
        return self.q

    def read(self, starts, lens, pages, stream=None):
        """The keys and values [T, Hkv, D] held for the call's tokens."""
        xhc_cache_read(self.d, self.h, self.c, *self._check(starts, lens, pages), self.pool, self.k, self.v, stream)
        return self.k, self.v

    def attend(self, q, starts, lens, pages, stream=None):
        """Attention of q [T, Hq, D], the call's tokens (appended before), over their sequences up to themselves."""
        q = _take(q, self.q.dtype, self.q.shape, self.device, "q")
        xhc_attn_cache(self.d, self.h, self.c, q, self.slopes, *self._check(starts, lens, pages), self.pool, self.out,
                       self.ws, stream)
        return self.out


def grad_tensors(grads):
    """The weight gradients of a backward, as a list: of a TrainableSublayer's
    or TrainableFlashGroup's dict, of the grads of a norm or block, or of a
    list of such.  The state's and the sublayer outputs' gradients, which flow
    on, are not among them."""
    if torch.is_tensor(grads):
        return [grads]
    if grads is None:
        return []
    if isinstance(grads, dict):
        return [t for n, v in grads.items() if n not in ("X", "F", "F_list", "dHres", "dHpost", "dp")
                for t in grad_tensors(v)]
    return [t for v in grads for t in grad_tensors(v)]


def clip_grad_norm(grads, max_norm, outs=None, stream=None):
    """Clips gradients by their global norm: out = g min(1, max_norm / (norm +
    1e-6)), in place unless ``outs`` (a list like ``grads``) is given; left as
    they are where the norm is not finite.  Returns the norm before the clip,
    an fp32 [1] tensor (nothing waits for it here)."""
    grads = list(grads)
    dev = _here(grads[0].device if grads else "cuda")
    for g in grads if outs is None else grads + list(outs):
        if g.get_device() != dev.index:
            raise ValueError(f"a gradient or output is on {g.device}, expected {dev}")
    with _within(stream):
        norm = torch.empty(1, dtype=torch.float32, device=dev)
        ws = torch.empty(xhc_grad_workspace_bytes(len(grads)), dtype=torch.uint8, device=dev)
    xhc_grad_clip(grads, max_norm, grads if outs is None else list(outs), norm, ws, stream)
    return norm
