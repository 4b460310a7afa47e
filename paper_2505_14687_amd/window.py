"""Token sequences: attention within a window (include/grat_window.h).

Marshalling only, in the manner of sequence.py: Q [B, Hq, N, d], K and V [B, Hkv, M, d] views (any strides with d contiguous); k_len (int32 [B]):
valid keys of each sequence; q_pos (int32 [B]): position of its first query, by default the queries are the newest tokens.

    O, lse = grat_window_attention_fwd(Q, K, V, scale, window=1024, sinks=4, return_lse=True)
    dQ, dK, dV = grat_window_attention_bwd(dO, Q, K, V, O, lse, scale, window=1024, sinks=4)

A query at position p sees the valid keys j <= p with p - j < window or j < sinks; with causal=False those with |p - j| < window or j < sinks.  window
None: no limit.  Nothing is recorded by autograd, and tensors that require a gradient are refused while it records: make the calls in a
torch.autograd.Function (examples/window_attention.py) or under torch.no_grad().
"""
from __future__ import annotations

import ctypes

import torch

from . import grat
from .grat import DTYPES, _f32, _i32, _i64, _on, _result, _vp, lib
from .sequence import (INT32_MAX, _check, _enter, _flat, _ints, _ps, _pt, _Sequence, _shared, _tensor)

_SIGNATURES = {
    "grat_window_attention_work": (_i64, [_ps, _i32, _i32, _i32]),
    "grat_window_attention_fwd": (_i32, [_ps] + [_pt] * 4 + [_vp, _f32, _i32, _i32, _vp, _vp]),
    "grat_window_attention_bwd": (_i32, [_ps] + [_pt] * 5 + [_vp] + [_pt] * 3 + [_f32, _i32, _i32, _vp, _vp]),
}
_lib = None
_native = None   # csrc/binding.cpp, as in grat.py; not None once _lib is not


class _NoNative:
    """In the place of _binding where that is not there: it takes no call."""
    window_fwd = window_bwd = staticmethod(lambda *args: None)


def _library() -> ctypes.CDLL:
    global _lib, _native
    if _lib is None:
        L = lib()
        for name, (result, arguments) in _SIGNATURES.items():
            getattr(L, name).restype = result
            getattr(L, name).argtypes = arguments
        native = grat._native
        if hasattr(native, "set_window_library"):
            native.set_window_library(*(ctypes.cast(getattr(L, name), _vp).value for name in _SIGNATURES))
        else:
            native = _NoNative
        _native = native   # (ahead of _lib: another thread that finds _lib set uses both)
        _lib = L
    return _lib


def _call(name: str, *args, written=()):
    _enter(_library(), name, args, written)


def _window(window, sinks) -> tuple:
    """Both as the library takes them: a window of 0 is none."""
    if window is not None and not 1 <= int(window) <= INT32_MAX:
        raise ValueError(f"window must be None or positive and at most {INT32_MAX}")
    if not 0 <= int(sinks) <= INT32_MAX:
        raise ValueError(f"sinks must not be negative and at most {INT32_MAX}")
    return 0 if window is None else int(window), int(sinks)


def _attention_args(Q, K, V, causal, k_len, q_pos) -> _Sequence:
    _check("Q", Q)
    _check("K", K, None, Q)
    B, Hq, N, d = Q.shape
    Hkv, M = K.shape[1], K.shape[2]
    _check("K", K, (B, Hkv, M, d), Q)
    _check("V", V, K.shape, Q)
    _shared(Hq, Hkv)
    return _Sequence(DTYPES[Q.dtype], B, Hq, Hkv, d, N, M, 0, 0, int(bool(causal)), _ints("k_len", k_len, B, Q.device),
                     _ints("q_pos", q_pos, B, Q.device))


def _work(need: int, device):
    return torch.empty(need, dtype=torch.uint8, device=device) if need else None


def _address(t):
    return None if t is None else t.data_ptr()


def grat_window_attention_fwd(Q, K, V, scale: float, window=None, sinks: int = 0, causal: bool = True, k_len=None, q_pos=None,
                              return_lse: bool = False, out=None, stream=None):
    """O = softmax(scale * Q K^T over the keys that a row sees) V; with return_lse also the rows' log-sum-exp, fp32 [B, Hq, N]."""
    _library()
    r = _native.window_fwd(Q, K, V, scale, window, sinks, causal, k_len, q_pos, return_lse, out, stream)
    if r is not None:
        return _result(r, "grat_window_attention_fwd")
    seq = _attention_args(Q, K, V, causal, k_len, q_pos)
    limits = _window(window, sinks)
    with _on(stream, Q.device) as s:
        work = _work(_lib.grat_window_attention_work(ctypes.byref(seq), *limits, 0), Q.device)
        O = torch.empty_like(Q) if out is None else out
        lse = torch.empty(Q.shape[:3], dtype=torch.float32, device=Q.device) if return_lse else None
        _check("out", O, Q.shape, Q)
        _call("grat_window_attention_fwd", ctypes.byref(seq), *(ctypes.byref(_tensor(t)) for t in (Q, K, V, O)), _address(lse), float(scale),
              *limits, _address(work), s, written=(out,))
    return (O, lse) if return_lse else O


def grat_window_attention_bwd(dO, Q, K, V, O, lse, scale: float, window=None, sinks: int = 0, causal: bool = True, k_len=None, q_pos=None,
                              out=None, stream=None):
    """(dQ, dK, dV) of grat_window_attention_fwd for dO; O and lse as it returned them.  out: three tensors to write to."""
    _library()
    r = _native.window_bwd(Q, K, V, scale, window, sinks, causal, k_len, q_pos, dO, O, lse, out, stream)
    if r is not None:
        return _result(r, "grat_window_attention_bwd")
    seq = _attention_args(Q, K, V, causal, k_len, q_pos)
    limits = _window(window, sinks)
    _check("dO", dO, Q.shape, Q)
    _check("O", O, Q.shape, Q)
    where = _flat("lse", lse, torch.float32, Q.shape[:3], Q.device)
    with _on(stream, Q.device) as s:
        work = _work(_lib.grat_window_attention_work(ctypes.byref(seq), *limits, 1), Q.device)
        dQ, dK, dV = grads = (torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V)) if out is None else tuple(out)
        for name, t, like in zip(("out[0]", "out[1]", "out[2]"), grads, (Q, K, V)):
            _check(name, t, like.shape, Q)
        _call("grat_window_attention_bwd", ctypes.byref(seq), *(ctypes.byref(_tensor(t)) for t in (dO, Q, K, V, O)), where,
              *(ctypes.byref(_tensor(t)) for t in (dQ, dK, dV)), float(scale), *limits, _address(work), s, written=() if out is None else grads)
    return dQ, dK, dV
