"""Token sequences: attention within a window, and over caches in 8 bits (include/grat_window.h).

Marshalling only, in the manner of sequence.py: Q [B, Hq, N, d], K and V [B, Hkv, M, d] views (any strides with d contiguous); k_len (int32 [B]):
valid keys of each sequence; q_pos (int32 [B]): position of its first query, by default the queries are the newest tokens.

    O, lse = grat_window_attention_fwd(Q, K, V, scale, window=1024, sinks=4, return_lse=True)
    dQ, dK, dV = grat_window_attention_bwd(dO, Q, K, V, O, lse, scale, window=1024, sinks=4)

    Q = grat_cache_append(Q, K, V, table, K_cache, V_cache, start, K_scale=K_scale, V_scale=V_scale)      # caches: float8_e4m3fn
    O = grat_cache_attention_fwd(Q, K_cache, V_cache, scale, k_len=start + n, K_scale=K_scale, V_scale=V_scale, parent=parent)
    K = grat_cache_read(K_cache, K_scale, torch.bfloat16)

A query at position p sees the valid keys j <= p with p - j < window or j < sinks; with causal=False those with |p - j| < window or j < sinks.  window
None: no limit.  Nothing is recorded by autograd, and tensors that require a gradient are refused while it records: make the calls in a
torch.autograd.Function (examples/window_attention.py) or under torch.no_grad().
"""
from __future__ import annotations

import ctypes

import torch

from . import grat
from .grat import DTYPES, _f32, _i32, _i64, _on, _result, _vp, lib
from .sequence import (INT32_MAX, LAYOUTS, _check, _enter, _flat, _ints, _no_gradient, _pr, _ps, _pt, _Rotary, _rotary_args, _Sequence, _shared,
                       _tensor, _Tensor)

EIGHT = torch.float8_e4m3fn
_SIGNATURES = {
    "grat_window_attention_work": (_i64, [_ps, _i32, _i32, _i32]),
    "grat_window_attention_fwd": (_i32, [_ps] + [_pt] * 4 + [_vp, _f32, _i32, _i32, _vp, _vp]),
    "grat_window_attention_bwd": (_i32, [_ps] + [_pt] * 5 + [_vp] + [_pt] * 3 + [_f32, _i32, _i32, _vp, _vp]),
    "grat_cache_append": (_i32, [_pr] + [_pt] * 8 + [_i32, _vp]),
    "grat_cache_read": (_i32, [_i32] * 5 + [_pt, _pt, _vp, _pt, _vp]),
    "grat_cache_attention_work": (_i64, [_ps, _i32, _i32, _i32]),
    "grat_cache_attention_fwd": (_i32, [_ps] + [_pt] * 6 + [_vp, _f32, _i32, _i32, _vp, _i64, _vp, _vp]),
}
_lib = None
_native = None   # csrc/binding.cpp, as in grat.py; not None once _lib is not


class _NoNative:
    """In the place of _binding where that is not there: it takes no call."""
    window_fwd = window_bwd = cache_append = cache_read = cache_attention = staticmethod(lambda *args: None)


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


# ---- caches -----------------------------------------------------------------------------------

def _check_cache(name: str, t, shape, like, scale) -> None:
    """A cache of the dtype of `like`, or of 8 bits beside its rows' scales."""
    if scale is None:
        _check(name, t, shape, like)
        return
    if not isinstance(t, torch.Tensor) or t.dtype != EIGHT:
        raise ValueError(f"{name} must be a tensor of {EIGHT}, beside its scales")
    if t.dim() != 4 or t.stride(3) != 1 or max(t.shape) > INT32_MAX:
        raise ValueError(f"{name}: expected a [B, H, N, d] tensor (any strides with d contiguous)")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {list(shape)}, not {list(t.shape)}")
    if not isinstance(scale, torch.Tensor) or scale.dtype != torch.float32 or tuple(scale.shape) != tuple(t.shape[:3]):
        raise ValueError(f"{name}'s scales must be float32 of shape {list(t.shape[:3])}")
    if (like is not None and t.device != like.device) or scale.device != t.device:
        raise ValueError(f"{name} and its scales must live on the tensors' device")
    _no_gradient(name, t)
    _no_gradient(f"{name}'s scales", scale)


def _scale(t):
    """float [B, H, N] as the library reads it."""
    if t is None:
        return None
    B, H, N = t.shape
    return ctypes.byref(_Tensor(t.data_ptr(), t.stride(0) if B > 1 else 0, t.stride(1) if H > 1 else 0, t.stride(2) if N > 1 else 1))


def _both(K_scale, V_scale) -> None:
    if (K_scale is None) != (V_scale is None):
        raise ValueError("K_scale and V_scale are given both (caches in 8 bits) or neither")


def grat_cache_append(Q, K, V, table, K_cache, V_cache, start, K_scale=None, V_scale=None, positions=None, layout: str = "half", axis_pairs=None,
                      out=None, stream=None):
    """Serving: returns Q turned, and writes K turned and V to rows start[b] + i of the caches.  Rows outside of them are dropped.

    With K_scale and V_scale (float32 [B, Hkv, M]) the caches are float8_e4m3fn, else of K's dtype.  positions int32 [B or 1, N, axes]: where a
    token's position is not its row (drafted trees).  Q None: K and V alone (returns None); table None: nothing is turned (then Q must be None)."""
    _library()
    r = _native.cache_append(Q, K, V, table, K_cache, V_cache, start, K_scale, V_scale, positions, LAYOUTS.get(layout), axis_pairs, out, stream)
    if r is not None:
        r = _result(r, "grat_cache_append")
        return None if Q is None else r
    _check("K", K)
    B, Hkv, N, d = K.shape
    if Q is not None:
        _check("Q", Q, (B, Q.shape[1] if isinstance(Q, torch.Tensor) and Q.dim() == 4 else 0, N, d), K)
    elif out is not None:
        raise ValueError("out is Q's: there is none")
    _check("V", V, K.shape, K)
    _both(K_scale, V_scale)
    _check_cache("K_cache", K_cache, None, K, K_scale)
    _check_cache("K_cache", K_cache, (B, Hkv, K_cache.shape[2], d), K, K_scale)
    _check_cache("V_cache", V_cache, K_cache.shape, K, V_scale)
    if start is None:
        raise ValueError("start must be given: tokens that each cache holds")
    if table is None:
        if Q is not None or positions is not None:
            raise ValueError("without a table nothing is turned: Q and positions must be None")
        if layout not in LAYOUTS:
            raise ValueError(f"layout must be one of {sorted(LAYOUTS)}")
        args = _Rotary(DTYPES[K.dtype], B, 0, Hkv, d, N, 0, 0, 0, 0, (_i32 * 3)(), None, 0, None, 0, None)
    else:
        args = _rotary_args(K if Q is None else Q, Hkv, table, positions, None, layout, axis_pairs, False)
    args.d_start = _ints("start", start, B, K.device)
    with _on(stream, K.device) as s:
        written = (K_cache, V_cache, K_scale, V_scale, out)
        if out is None and Q is not None:
            out = torch.empty_like(Q)
        if Q is not None:
            _check("out", out, Q.shape, Q)
        q = (None, None) if Q is None else (ctypes.byref(_tensor(Q)), ctypes.byref(_tensor(out)))
        _call("grat_cache_append", ctypes.byref(args), *q, *(ctypes.byref(_tensor(t)) for t in (K, V, K_cache, V_cache)), _scale(K_scale),
              _scale(V_scale), int(K_cache.shape[2]), s, written=written)
    return out


def grat_cache_read(cache, scale, dtype, k_len=None, out=None, stream=None):
    """A cache of float8_e4m3fn rows and their scales (float32 [B, H, N]) in dtype, [B, H, N, d]; rows behind k_len get 0."""
    _library()
    r = _native.cache_read(cache, scale, DTYPES.get(dtype), k_len, out, stream)
    if r is not None:
        return _result(r, "grat_cache_read")
    if dtype not in DTYPES:
        raise ValueError(f"unsupported dtype {dtype}")
    if scale is None:
        raise ValueError("scale must be given")
    _check_cache("cache", cache, None, None, scale)
    B, H, N, d = cache.shape
    lengths = _ints("k_len", k_len, B, cache.device)
    with _on(stream, cache.device) as s:
        written = (out,)
        if out is None:
            out = torch.empty(cache.shape, dtype=dtype, device=cache.device)
        _check("out", out, cache.shape)
        if out.dtype != dtype or out.device != cache.device:
            raise ValueError("out must have the given dtype and the cache's device")
        _call("grat_cache_read", DTYPES[dtype], B, H, N, d, ctypes.byref(_tensor(cache)), _scale(scale), lengths, ctypes.byref(_tensor(out)), s,
              written=written)
    return out


def grat_cache_attention_fwd(Q, K_cache, V_cache, scale: float, k_len=None, K_scale=None, V_scale=None, parent=None, window=None, sinks: int = 0,
                             return_lse: bool = False, out=None, stream=None):
    """O of the newest tokens over a cache that holds their K and V in its rows [k_len - N, k_len), in Q's dtype or, with K_scale and V_scale, in 8 bits.

    parent int32 [N], [1, N] or [B, N]: a tree.  Token t goes on from token parent[t] < t, or (-1) from the newest committed token, and sees the
    committed tokens, its ancestors and itself; its position is k_len - N + its depth.  None: a chain.  window, sinks: as for
    grat_window_attention_fwd, by positions.  With return_lse also the rows' log-sum-exp, fp32 [B, Hq, N]."""
    _library()
    r = _native.cache_attention(Q, K_cache, V_cache, scale, k_len, K_scale, V_scale, parent, window, sinks, return_lse, out, stream)
    if r is not None:
        return _result(r, "grat_cache_attention_fwd")
    _check("Q", Q)
    B, Hq, N, d = Q.shape
    _both(K_scale, V_scale)
    _check_cache("K_cache", K_cache, None, Q, K_scale)
    Hkv, M = K_cache.shape[1], K_cache.shape[2]
    _check_cache("K_cache", K_cache, (B, Hkv, M, d), Q, K_scale)
    _check_cache("V_cache", V_cache, K_cache.shape, Q, V_scale)
    _shared(Hq, Hkv)
    limits, eight = _window(window, sinks), K_scale is not None
    line, line_stride = None, 0
    if parent is not None:
        if isinstance(parent, torch.Tensor) and parent.dim() == 1:
            parent = parent.unsqueeze(0)
        if not isinstance(parent, torch.Tensor) or parent.dim() != 2 or parent.shape[0] not in (1, B):
            raise ValueError(f"parent must be int32 [{N}], or [{B} or 1, {N}]")
        line = _flat("parent", parent, torch.int32, (parent.shape[0], N), Q.device)
        line_stride = N if parent.shape[0] > 1 else 0
    seq = _Sequence(DTYPES[Q.dtype], B, Hq, Hkv, d, N, M, 0, 0, 1, _ints("k_len", k_len, B, Q.device), None)
    with _on(stream, Q.device) as s:
        work = _work(_lib.grat_cache_attention_work(ctypes.byref(seq), *limits, int(eight)), Q.device)
        O = torch.empty_like(Q) if out is None else out
        lse = torch.empty(Q.shape[:3], dtype=torch.float32, device=Q.device) if return_lse else None
        _check("out", O, Q.shape, Q)
        _call("grat_cache_attention_fwd", ctypes.byref(seq), *(ctypes.byref(_tensor(t)) for t in (Q, K_cache, V_cache)), _scale(K_scale),
              _scale(V_scale), ctypes.byref(_tensor(O)), _address(lse), float(scale), *limits, line, line_stride, _address(work), s, written=(out,))
    return (O, lse) if return_lse else O
