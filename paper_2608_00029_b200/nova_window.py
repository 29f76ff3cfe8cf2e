"""Binding of the attention with a sliding window and sinks of libnova_attn.so (include/nova_window.h): argument checks and
marshalling only.  No CPU fallback: a missing library or a failed call raises.  Calls run on the device of their tensors.

Query i keeps key j if j <= i and (i - j < window or j < sinks).  Tensors are [B,H,T,D]-shaped bf16 views, strides taken from
them; K, V and their gradients may have fewer heads than Q, a divisor."""
from __future__ import annotations

import ctypes
import operator

from . import nova_attn as _na

_ready = False


def _lib():
    global _ready
    lib = _na.load()
    if not _ready:
        i, sz = ctypes.c_int, ctypes.c_size_t
        for f in (lib.nova_window_bwd_workspace_bytes, lib.nova_window_decode_workspace_bytes):
            f.argtypes = [i] * 7
            f.restype = sz
        _ready = True
    return lib


def _ints(**named):
    """Whole numbers that fit the C ABI's int, in order."""
    for name, x in named.items():
        if not -2**31 <= operator.index(x) < 2**31:
            raise ValueError(f"{name} is out of range")
    return [operator.index(x) for x in named.values()]


def nova_window_fwd(Q, K, V, O, LSE, scale: float, window: int, sinks: int = 0, O_rest=None, stream=None) -> None:
    """O, LSE <- attention(Q, K, V); LSE is contiguous fp32 [B,H,T].  O_rest (strides of O): what rounding took from O, for
    nova_window_bwd_preprocess."""
    rc = _na._binding().window_fwd(Q, K, V, O, O_rest, LSE, scale, window, sinks, stream)
    if rc != _na.OK:
        raise _na.NovaAttnError(rc, "nova_window_fwd")


def nova_window_bwd_preprocess(O, O_rest, dO, Delta, stream=None) -> None:
    """Delta <- rowsum(dO * (O + O_rest)); O_rest may be None, at the price of the rounding of O in dQ and dK."""
    rc = _na._binding().window_preprocess(O, O_rest, dO, Delta, stream)
    if rc != _na.OK:
        raise _na.NovaAttnError(rc, "nova_window_bwd_preprocess")


def nova_window_bwd_workspace_bytes(B: int, H: int, H_kv: int, T: int, D: int, window: int, sinks: int = 0) -> int:
    return int(_lib().nova_window_bwd_workspace_bytes(*_ints(B=B, H=H, H_kv=H_kv, T=T, D=D, window=window, sinks=sinks)))


def nova_window_bwd(Q, K, V, dO, LSE, Delta, dQ, dK, dV, scale: float, window: int, sinks: int = 0, workspace=None,
                    stream=None) -> None:
    """dQ, dK, dV <- gradients of sum(O*dO), bitwise reproducible; `workspace` is a CUDA tensor without gaps of at least
    nova_window_bwd_workspace_bytes(B,H,H_kv,T,D,window,sinks) bytes (allocated here if omitted)."""
    rc = _na._binding().window_bwd(Q, K, V, dO, LSE, Delta, dQ, dK, dV, scale, window, sinks, workspace, stream)
    if rc != _na.OK:
        raise _na.NovaAttnError(rc, "nova_window_bwd")


def nova_window_decode_workspace_bytes(B: int, H: int, H_kv: int, T_max: int, D: int, window: int, sinks: int = 0) -> int:
    return int(_lib().nova_window_decode_workspace_bytes(*_ints(B=B, H=H, H_kv=H_kv, T_max=T_max, D=D, window=window, sinks=sinks)))


def nova_window_decode(Q, K, V, lengths, O, LSE, scale: float, window: int, sinks: int = 0, workspace=None, stream=None) -> None:
    """One new token per sequence: O [B,H,1,D], LSE [B,H,1] <- the last row of the attention of Q [B,H,1,D] over the first
    lengths[b] (int32 on the GPU) tokens of the caches K, V [B,H_kv,T_max,D], the new token among them.  A sequence of length 0
    gets O = 0, LSE = -inf.  `workspace` as in nova_window_bwd, nova_window_decode_workspace_bytes(...) bytes."""
    rc = _na._binding().window_decode(Q, K, V, lengths, O, LSE, scale, window, sinks, workspace, stream)
    if rc != _na.OK:
        raise _na.NovaAttnError(rc, "nova_window_decode")
