"""Binding of the rotary positions of libnova_attn.so (include/nova_rope.h): argument checks and marshalling only.  No CPU
fallback: a missing library or a failed call raises.  Calls run on the device of their tensors."""
from __future__ import annotations

import ctypes
import operator

import torch

from . import nova_attn as _na

_ready = False
_KINDS = {"plain": 0, "linear": 1, "base": 2, "bands": 3, "yarn": 4}


def _lib():
    global _ready
    lib = _na.load()
    if not _ready:
        i, d = ctypes.c_int, ctypes.c_double
        f = ctypes.POINTER(ctypes.c_float)
        lib.nova_rope_frequencies.argtypes = [f, f, i, d, i, d, ctypes.c_longlong, d, d]
        lib.nova_rope_frequencies.restype = i
        _ready = True
    return lib


def nova_rope_frequencies(rotary: int, base: float = 10000.0, kind: str = "plain", factor: float = 1.0, original: int = 0,
                          low: float = 1.0, high: float = 32.0):
    """(inv_freq, amplitude) of a model: inv_freq a CPU fp32 tensor [rotary / 2], amplitude a float.  `kind` says how the
    frequencies are scaled for a context `factor` times as long as the `original` positions: "plain", "linear", "base",
    "bands" or "yarn" (`low` and `high` turns bound the last two's bands), as in the header."""
    if kind not in _KINDS:
        raise ValueError(f"kind must be one of {', '.join(_KINDS)}, not {kind!r}")
    rotary, original = operator.index(rotary), operator.index(original)
    if not -2**31 <= rotary < 2**31 or not -2**63 <= original < 2**63:
        raise ValueError("rotary or original is out of range")
    freq = (ctypes.c_float * max(1, rotary // 2))()
    amplitude = ctypes.c_float()
    rc = _lib().nova_rope_frequencies(freq, ctypes.byref(amplitude), rotary, float(base), _KINDS[kind], float(factor), original,
                                      float(low), float(high))
    if rc != _na.OK:
        raise _na.NovaAttnError(rc, "nova_rope_frequencies")
    return torch.tensor(list(freq), dtype=torch.float32), float(amplitude.value)


def nova_rope_fwd(Q, K, Q_out, K_out, inv_freq, positions=None, interleaved: bool = False, amplitude: float = 1.0,
                  stream=None) -> None:
    """Q_out, K_out <- Q, K turned by their tokens' positions.  Q, Q_out [B,H,T,D] and K, K_out [B,H_kv,T,D] are bf16 views
    (strides are taken from the tensors, slices of a fused projection output are fine, and Q_out may be Q and K_out K); K and
    K_out may both be None.  inv_freq: fp32 [rotary / 2] on the GPU, pairs (i, i + rotary/2), or (2i, 2i+1) if `interleaved`;
    positions: int32 [T] or [B,T] on the GPU, None for 0 .. T-1."""
    rc = _na._binding().rope(Q, K, Q_out, K_out, inv_freq, positions, interleaved, amplitude, False, stream)
    if rc != _na.OK:
        raise _na.NovaAttnError(rc, "nova_rope_fwd")


def nova_rope_bwd(dQ_out, dK_out, dQ, dK, inv_freq, positions=None, interleaved: bool = False, amplitude: float = 1.0,
                  stream=None) -> None:
    """dQ, dK <- gradients of Q and K of nova_rope_fwd from those of Q_out and K_out; arguments as there."""
    rc = _na._binding().rope(dQ_out, dK_out, dQ, dK, inv_freq, positions, interleaved, amplitude, True, stream)
    if rc != _na.OK:
        raise _na.NovaAttnError(rc, "nova_rope_bwd")
