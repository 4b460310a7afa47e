"""Token sequences: rotary positions, and attention over key blocks that a score selects (include/grat_sequence.h).

Marshalling only, like grat.py (ordinary calls on the current stream in csrc/binding.cpp, all others here): every step runs in the
library's kernels, on the tensors' device, on its current stream or the one that is given.  Results and scratch memory are allocated for the stream that the call runs on.

    table = grat_rotary_table(n_pos, [head_dim // 2])                      # once
    Q, K = grat_rotary(Q, K, table)
    means = grat_block_means(K, block)
    scores = grat_block_scores(Q, means, scale, q_group, block, n_k=K.shape[2])
    count, index = grat_select_blocks(scores, top, first=1, local=2, n_q=Q.shape[2], n_k=K.shape[2], q_group=q_group, block=block)
    O = grat_selected_attention_fwd(Q, K, V, scale, count, index, q_group, block)

Q is [B, Hq, N, d], K and V are [B, Hkv, M, d] views (any strides with d contiguous); Hkv divides Hq.  k_len (int32 [B]): valid keys of
each sequence; q_pos (int32 [B]): position of its first query, by default the queries are the newest tokens.

Nothing is recorded by autograd, and tensors that require a gradient are refused while it records: make the calls in a torch.autograd.Function
(examples/selected_attention.py), with grat_rotary(inverse=True) and grat_selected_attention_bwd in its backward, or under torch.no_grad().
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch
from torch.autograd import forward_ad

from . import grat
from .grat import DTYPES, GRAT_OK, GratError, _i32, _i64, _f32, _on, _result, _vp, lib

SCALINGS = {"plain": 0, "linear": 1, "base": 2, "ramp": 3}
LAYOUTS = {"half": 0, "interleaved": 1}
INT32_MAX = 2 ** 31 - 1   # the library's sizes; what is beyond would be cut off on the way


class _Tensor(ctypes.Structure):
    _fields_ = [("data", _vp), ("stride_b", _i64), ("stride_h", _i64), ("stride_n", _i64)]


class _Sequence(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("batch", _i32), ("q_heads", _i32), ("kv_heads", _i32), ("head_dim", _i32), ("n_q", _i32),
                ("n_k", _i32), ("q_group", _i32), ("block", _i32), ("causal", _i32), ("d_k_len", _vp), ("d_q_pos", _vp)]


class _Rotary(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("batch", _i32), ("q_heads", _i32), ("kv_heads", _i32), ("head_dim", _i32), ("n_tokens", _i32),
                ("rot", _i32), ("interleaved", _i32), ("inverse", _i32), ("axes", _i32), ("axis_pairs", _i32 * 3), ("d_table", _vp),
                ("n_pos", _i32), ("d_positions", _vp), ("positions_stride_b", _i64), ("d_start", _vp)]


class _Spec(ctypes.Structure):
    _fields_ = [("scaling", _i32)] + [(n, ctypes.c_double) for n in ("base", "factor", "magnitude", "trained", "low", "high")]


_pt, _ps, _pr = ctypes.POINTER(_Tensor), ctypes.POINTER(_Sequence), ctypes.POINTER(_Rotary)
_SIGNATURES = {
    "grat_rotary_table": (_i32, [ctypes.POINTER(_Spec), _i32, _i32, ctypes.POINTER(_i32), _vp, _vp]),
    "grat_rotary": (_i32, [_pr, _pt, _pt, _pt, _pt, _vp]),
    "grat_rotary_append": (_i32, [_pr, _pt, _pt, _pt, _pt, _pt, _pt, _i32, _vp]),
    "grat_block_means": (_i32, [_ps, _pt, _i32, _vp, _vp]),
    "grat_block_scores_work": (_i64, [_ps]),
    "grat_block_scores": (_i32, [_ps, _pt, _vp, _f32, _vp, _vp, _vp]),
    "grat_select_blocks": (_i32, [_ps, _vp, _i32, _i32, _i32, _vp, _vp, _vp]),
    "grat_selected_attention_work": (_i64, [_ps, _i32, _i32]),
    "grat_selected_attention_fwd": (_i32, [_ps, _pt, _pt, _pt, _pt, _vp, _f32, _vp, _vp, _i32, _vp, _vp]),
    "grat_selected_attention_bwd": (_i32, [_ps] + [_pt] * 5 + [_vp] + [_pt] * 3 + [_f32, _vp, _vp, _i32, _vp, _vp]),
}
_lib = None
_native = None   # csrc/binding.cpp, as in grat.py; not None once _lib is not


class _NoNative:
    """In the place of _binding where that is not there: it takes no call."""
    rotary = append = means = scores = select = selected_fwd = selected_bwd = staticmethod(lambda *args: None)


def _library() -> ctypes.CDLL:
    global _lib, _native
    if _lib is None:
        L = lib()
        for name, (result, arguments) in _SIGNATURES.items():
            getattr(L, name).restype = result
            getattr(L, name).argtypes = arguments
        native = grat._native
        if hasattr(native, "set_sequence_library"):
            native.set_sequence_library(*(ctypes.cast(getattr(L, name), _vp).value for name in _SIGNATURES if name != "grat_rotary_table"))
        else:
            native = _NoNative
        _native = native   # (ahead of _lib: another thread that finds _lib set uses both)
        _lib = L
    return _lib


def _call(name: str, *args, written=()):
    _enter(_library(), name, args, written)


def _enter(L: ctypes.CDLL, name: str, args, written):
    """written: the caller's tensors that it writes to; autograd then notices where it had saved one of them."""
    st = getattr(L, name)(*args)
    if st != GRAT_OK:
        raise GratError(st, name)
    for t in written:
        if t is not None and not t.is_inference():   # (these have no version)
            torch.autograd.graph.increment_version(t)


def _tensor(t: torch.Tensor) -> _Tensor:
    B, H, N, d = t.shape   # (the stride of an axis of one element counts for nothing and may be any number)
    return _Tensor(t.data_ptr(), t.stride(0) if B > 1 else 0, t.stride(1) if H > 1 else 0, t.stride(2) if N > 1 else d)


def _no_gradient(name: str, t) -> None:
    """What the library computes is not recorded by autograd: the gradient of such a tensor would be lost without a word."""
    if torch.is_grad_enabled() and t.requires_grad or forward_ad.unpack_dual(t).tangent is not None:
        raise ValueError(f"{name} requires a gradient, which these calls do not record: make them in a torch.autograd.Function whose backward "
                         "calls the gradients' entry points, or under torch.no_grad()")


def _check(name: str, t, shape=None, like=None):
    """A [B, H, N, d] tensor as the library reads it."""
    if not isinstance(t, torch.Tensor) or t.dim() != 4:
        raise ValueError(f"{name}: expected a [B, H, N, d] tensor (any strides with d contiguous)")
    if t.stride(3) != 1:
        raise ValueError(f"{name}: the head_dim axis must be contiguous")
    if max(t.shape) > INT32_MAX:
        raise ValueError(f"{name}: an axis is longer than {INT32_MAX}")
    if t.dtype not in DTYPES:
        raise ValueError(f"{name}: unsupported dtype {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {list(shape)}, not {list(t.shape)}")
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        raise ValueError(f"{name} must have the dtype and the device of the other tensors")
    _no_gradient(name, t)


def _flat(name: str, t, dtype, shape, device, differentiable: bool = True) -> int:
    """A contiguous tensor of one shape; its address."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype:
        raise ValueError(f"{name} must be a tensor of {dtype}")
    if tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous and have shape {list(shape)}, not {list(t.shape)}")
    if t.device != device:
        raise ValueError(f"{name} must live on the tensors' device ({device})")
    if differentiable:
        _no_gradient(name, t)
    return t.data_ptr()


def _ints(name: str, t, batch: int, device) -> Optional[int]:
    return None if t is None else _flat(name, t, torch.int32, (batch,), device)


def _positive(**values) -> None:
    for name, v in values.items():
        if not 1 <= int(v) <= INT32_MAX:
            raise ValueError(f"{name} must be positive and at most {INT32_MAX}")


def _int32(**values) -> None:   # (the library refuses what is negative)
    for name, v in values.items():
        if abs(int(v)) > INT32_MAX:
            raise ValueError(f"{name} must be at most {INT32_MAX}")


def _shared(q_heads: int, kv_heads: int) -> None:
    if kv_heads < 1 or q_heads % kv_heads:
        raise ValueError(f"{q_heads} query heads cannot share {kv_heads} K/V heads")


def _ceil(a: int, b: int) -> int:
    return -(-a // b)


# ---- rotary positions -------------------------------------------------------------------------

def grat_rotary_table(n_pos: int, axis_pairs: Sequence[int], base: float = 10000.0, scaling: str = "plain", factor: float = 1.0,
                      magnitude: float = 1.0, trained: float = 0.0, low: float = 1.0, high: float = 32.0, device="cuda", stream=None):
    """cos and sin of every position and pair, fp32 [n_pos, pairs, 2].  axis_pairs: pairs of every axis, [rot // 2] for a sequence."""
    pairs = [int(p) for p in axis_pairs]
    if scaling not in SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(SCALINGS)}")
    _positive(n_pos=n_pos)
    if not 1 <= len(pairs) <= 3 or min(pairs) < 1 or max(pairs) > INT32_MAX:
        raise ValueError("axis_pairs must hold 1 to 3 positive numbers")
    device = torch.device(device)
    spec = _Spec(SCALINGS[scaling], float(base), float(factor), float(magnitude), float(trained), float(low), float(high))
    with _on(stream, device) as s:
        table = torch.empty((int(n_pos), sum(pairs), 2), dtype=torch.float32, device=device)
        _call("grat_rotary_table", ctypes.byref(spec), int(n_pos), len(pairs), (_i32 * len(pairs))(*pairs), table.data_ptr(), s)
    return table


def _rotary_args(Q, kv_heads: int, table, positions, start, layout: str, axis_pairs, inverse: bool) -> _Rotary:
    B, H, N, d = Q.shape
    if layout not in LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(LAYOUTS)}")
    if not isinstance(table, torch.Tensor) or table.dim() != 3 or table.shape[2] != 2:
        raise ValueError("table must have shape [n_pos, rot / 2, 2]")
    where = _flat("table", table, torch.float32, table.shape, Q.device)
    pairs = [int(table.shape[1])] if axis_pairs is None else [int(p) for p in axis_pairs]
    if not 1 <= len(pairs) <= 3 or min(pairs) < 1 or sum(pairs) != table.shape[1]:
        raise ValueError("axis_pairs must hold 1 to 3 positive numbers that add up to the table's pairs")
    if 2 * table.shape[1] > d:
        raise ValueError("the table has more pairs than a head")
    if table.shape[0] > INT32_MAX:
        raise ValueError(f"the table has more than {INT32_MAX} positions")
    if positions is not None and start is not None:
        raise ValueError("positions and start exclude each other")
    at, stride = None, 0
    if positions is not None:
        axes = len(pairs)
        if isinstance(positions, torch.Tensor) and positions.dim() == 2 and axes == 1:
            positions = positions.unsqueeze(-1)
        if not isinstance(positions, torch.Tensor) or positions.dim() != 3 or positions.shape[0] not in (1, B):
            raise ValueError(f"positions must be int32 [{B} or 1, {N}, {axes}]")
        at = _flat("positions", positions, torch.int32, (positions.shape[0], N, axes), Q.device)
        stride = N * axes if positions.shape[0] > 1 else 0
    elif len(pairs) > 1:
        raise ValueError("several axes need positions")
    return _Rotary(DTYPES[Q.dtype], B, H, kv_heads, d, N, 2 * table.shape[1], LAYOUTS[layout], int(bool(inverse)), len(pairs),
                   (_i32 * 3)(*pairs), where, int(table.shape[0]), at, stride, _ints("start", start, B, Q.device))


def grat_rotary(Q, K, table, positions=None, start=None, layout: str = "half", axis_pairs: Optional[Sequence[int]] = None,
                inverse: bool = False, out=None, stream=None):
    """Q and K (or None) turned by their positions; returns both (K's place None where K is).

    positions int32 [B or 1, N, axes], or start int32 [B] (token i is at start + i), or neither (token i is at i).  inverse: the
    gradient.  out: a pair of tensors to write to; Q and K themselves for a rotation in place."""
    _library()
    r = _native.rotary(Q, K, table, positions, start, LAYOUTS.get(layout), axis_pairs, inverse, out, stream)
    if r is not None:
        return _result(r, "grat_rotary")
    _check("Q", Q)
    if K is not None:
        _check("K", K, (Q.shape[0], K.shape[1] if isinstance(K, torch.Tensor) and K.dim() == 4 else 0, Q.shape[2], Q.shape[3]), Q)
    args = _rotary_args(Q, 0 if K is None else K.shape[1], table, positions, start, layout, axis_pairs, inverse)
    with _on(stream, Q.device) as s:
        written = () if out is None else tuple(out)
        if out is None:
            out = torch.empty_like(Q), None if K is None else torch.empty_like(K)
        Qo, Ko = out
        _check("out[0]", Qo, Q.shape, Q)
        if K is not None:
            _check("out[1]", Ko, K.shape, Q)
        k = (None, None) if K is None else (ctypes.byref(_tensor(K)), ctypes.byref(_tensor(Ko)))
        _call("grat_rotary", ctypes.byref(args), ctypes.byref(_tensor(Q)), ctypes.byref(_tensor(Qo)), *k, s, written=written[:1 if K is None else 2])
    return Qo, Ko


def grat_rotary_append(Q, K, V, table, K_cache, V_cache, start, layout: str = "half", out=None, stream=None):
    """Serving: returns Q turned, and writes K turned and V to rows start[b] + i of the caches.  Rows outside of them are dropped."""
    _library()
    r = _native.append(Q, K, V, table, K_cache, V_cache, start, LAYOUTS.get(layout), out, stream)
    if r is not None:
        return _result(r, "grat_rotary_append")
    _check("Q", Q)
    _check("K", K, None, Q)
    B, _, N, d = Q.shape
    _check("K", K, (B, K.shape[1], N, d), Q)
    _check("V", V, K.shape, Q)
    _check("K_cache", K_cache, None, Q)
    _check("K_cache", K_cache, (B, K.shape[1], K_cache.shape[2], d), Q)
    _check("V_cache", V_cache, K_cache.shape, Q)
    if start is None:
        raise ValueError("start must be given: tokens that each cache holds")
    args = _rotary_args(Q, K.shape[1], table, None, start, layout, None, False)
    with _on(stream, Q.device) as s:
        written = (K_cache, V_cache, out)
        if out is None:
            out = torch.empty_like(Q)
        _check("out", out, Q.shape, Q)
        _call("grat_rotary_append", ctypes.byref(args), *(ctypes.byref(_tensor(t)) for t in (Q, out, K, V, K_cache, V_cache)),
              int(K_cache.shape[2]), s, written=written)
    return out


# ---- lists ------------------------------------------------------------------------------------

def grat_block_means(K, block: int, k_len=None, new: int = 0, out=None, stream=None):
    """Mean of the valid keys of every block, fp32 [B, Hkv, blocks, d].  new > 0: only the blocks with one of the last `new` valid
    keys are written, to `out`, which holds the others."""
    _library()
    r = _native.means(K, block, k_len, new, out, stream)
    if r is not None:
        return _result(r, "grat_block_means")
    _check("K", K)
    _positive(block=block)
    _int32(new=new)
    B, H, M, d = K.shape
    if int(new) < 0 or (int(new) > 0 and out is None):
        raise ValueError("new keys are added to means that are given as out")
    shape = (B, H, _ceil(M, int(block)), d)
    seq = _Sequence(DTYPES[K.dtype], B, H, H, d, 1, M, 1, int(block), 0, _ints("k_len", k_len, B, K.device), None)
    with _on(stream, K.device) as s:
        written = (out,)
        if out is None:
            out = torch.empty(shape, dtype=torch.float32, device=K.device)
        _call("grat_block_means", ctypes.byref(seq), ctypes.byref(_tensor(K)), int(new), _flat("out", out, torch.float32, shape, K.device), s,
              written=written)
    return out


def grat_block_scores(Q, means, scale: float, q_group: int, block: int, n_k: int, causal: bool = True, k_len=None, q_pos=None,
                      out=None, stream=None):
    """Score of every query group for every key block, fp32 [B, Hkv, groups, blocks]; -inf for blocks that a group does not see."""
    _library()
    r = _native.scores(Q, means, scale, q_group, block, n_k, causal, k_len, q_pos, out, stream)
    if r is not None:
        return _result(r, "grat_block_scores")
    _check("Q", Q)
    _positive(q_group=q_group, block=block, n_k=n_k)
    B, Hq, N, d = Q.shape
    if not isinstance(means, torch.Tensor) or means.dim() != 4:
        raise ValueError("means must have shape [B, Hkv, blocks, d]")
    Hkv, blocks, groups = means.shape[1], _ceil(int(n_k), int(block)), _ceil(N, int(q_group))
    _shared(Hq, Hkv)
    where = _flat("means", means, torch.float32, (B, Hkv, blocks, d), Q.device)
    seq = _Sequence(DTYPES[Q.dtype], B, Hq, Hkv, d, N, int(n_k), int(q_group), int(block), int(bool(causal)),
                    _ints("k_len", k_len, B, Q.device), _ints("q_pos", q_pos, B, Q.device))
    need = _lib.grat_block_scores_work(ctypes.byref(seq))
    with _on(stream, Q.device) as s:
        work, written = torch.empty(need, dtype=torch.uint8, device=Q.device) if need else None, (out,)
        if out is None:
            out = torch.empty((B, Hkv, groups, blocks), dtype=torch.float32, device=Q.device)
        _call("grat_block_scores", ctypes.byref(seq), ctypes.byref(_tensor(Q)), where, float(scale),
              _flat("out", out, torch.float32, (B, Hkv, groups, blocks), Q.device), work.data_ptr() if need else None, s, written=written)
    return out


def grat_select_blocks(scores, top: int, first: int, local: int, n_q: int, n_k: int, q_group: int, block: int, causal: bool = True,
                       k_len=None, q_pos=None, stream=None):
    """The lists: (count int32 [B, Hkv, groups], index int32 [B, Hkv, groups, top]), ascending, -1 behind a list's end.

    The choice of a group's blocks depends on all of its queries, up to q_group - 1 of them later than a row's own; with q_group 1 and
    local >= 1 on no later token."""
    _library()
    r = _native.select(scores, top, first, local, n_q, n_k, q_group, block, causal, k_len, q_pos, stream)
    if r is not None:
        return _result(r, "grat_select_blocks")
    _positive(top=top, n_q=n_q, n_k=n_k, q_group=q_group, block=block)
    _int32(first=first, local=local)
    if not isinstance(scores, torch.Tensor) or scores.dim() != 4:
        raise ValueError("scores must have shape [B, Hkv, groups, blocks]")
    B, Hkv, groups, blocks = scores.shape
    where = _flat("scores", scores, torch.float32, (B, Hkv, _ceil(int(n_q), int(q_group)), _ceil(int(n_k), int(block))), scores.device,
                  differentiable=False)   # (the lists are whole numbers)
    seq = _Sequence(0, B, Hkv, Hkv, 0, int(n_q), int(n_k), int(q_group), int(block), int(bool(causal)),
                    _ints("k_len", k_len, B, scores.device), _ints("q_pos", q_pos, B, scores.device))
    with _on(stream, scores.device) as s:
        count = torch.empty((B, Hkv, groups), dtype=torch.int32, device=scores.device)
        index = torch.empty((B, Hkv, groups, int(top)), dtype=torch.int32, device=scores.device)
        _call("grat_select_blocks", ctypes.byref(seq), where, int(top), int(first), int(local), count.data_ptr(), index.data_ptr(), s)
    return count, index


# ---- attention --------------------------------------------------------------------------------

def _attention_args(Q, K, V, count, index, q_group, block, causal, k_len, q_pos):
    _check("Q", Q)
    _check("K", K, None, Q)
    _positive(q_group=q_group, block=block)
    B, Hq, N, d = Q.shape
    Hkv, M = K.shape[1], K.shape[2]
    _check("K", K, (B, Hkv, M, d), Q)
    _check("V", V, K.shape, Q)
    _shared(Hq, Hkv)
    groups = _ceil(N, int(q_group))
    if not isinstance(index, torch.Tensor) or index.dim() != 4 or index.shape[3] < 1:
        raise ValueError(f"index must have shape [{B}, {Hkv}, {groups}, top]")
    lists = (_flat("count", count, torch.int32, (B, Hkv, groups), Q.device),
             _flat("index", index, torch.int32, (B, Hkv, groups, index.shape[3]), Q.device), int(index.shape[3]))
    seq = _Sequence(DTYPES[Q.dtype], B, Hq, Hkv, d, N, M, int(q_group), int(block), int(bool(causal)),
                    _ints("k_len", k_len, B, Q.device), _ints("q_pos", q_pos, B, Q.device))
    return seq, lists


def _work(seq: _Sequence, top: int, backward: int, device):
    need = _lib.grat_selected_attention_work(ctypes.byref(seq), top, backward)
    return torch.empty(need, dtype=torch.uint8, device=device) if need else None


def grat_selected_attention_fwd(Q, K, V, scale: float, count, index, q_group: int, block: int, causal: bool = True, k_len=None,
                                q_pos=None, return_lse: bool = False, out=None, stream=None):
    """O = softmax(scale * Q K^T over the listed keys that a row sees) V; with return_lse also the rows' log-sum-exp, fp32 [B, Hq, N]."""
    _library()
    r = _native.selected_fwd(Q, K, V, scale, count, index, q_group, block, causal, k_len, q_pos, return_lse, out, stream)
    if r is not None:
        return _result(r, "grat_selected_attention_fwd")
    seq, lists = _attention_args(Q, K, V, count, index, q_group, block, causal, k_len, q_pos)
    with _on(stream, Q.device) as s:
        work = _work(seq, lists[2], 0, Q.device)
        O = torch.empty_like(Q) if out is None else out
        lse = torch.empty(Q.shape[:3], dtype=torch.float32, device=Q.device) if return_lse else None
        _check("out", O, Q.shape, Q)
        _call("grat_selected_attention_fwd", ctypes.byref(seq), *(ctypes.byref(_tensor(t)) for t in (Q, K, V, O)),
              lse.data_ptr() if return_lse else None, float(scale), *lists, work.data_ptr() if work is not None else None, s,
              written=(out,))
    return (O, lse) if return_lse else O


def grat_selected_attention_bwd(dO, Q, K, V, O, lse, scale: float, count, index, q_group: int, block: int, causal: bool = True,
                                k_len=None, q_pos=None, out=None, stream=None):
    """(dQ, dK, dV) of grat_selected_attention_fwd for dO; O and lse as it returned them.  out: three tensors to write to."""
    _library()
    r = _native.selected_bwd(Q, K, V, scale, count, index, q_group, block, causal, k_len, q_pos, dO, O, lse, out, stream)
    if r is not None:
        return _result(r, "grat_selected_attention_bwd")
    seq, lists = _attention_args(Q, K, V, count, index, q_group, block, causal, k_len, q_pos)
    _check("dO", dO, Q.shape, Q)
    _check("O", O, Q.shape, Q)
    where = _flat("lse", lse, torch.float32, Q.shape[:3], Q.device)
    with _on(stream, Q.device) as s:
        work = _work(seq, lists[2], 1, Q.device)
        dQ, dK, dV = grads = (torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V)) if out is None else tuple(out)
        for name, t, like in zip(("out[0]", "out[1]", "out[2]"), grads, (Q, K, V)):
            _check(name, t, like.shape, Q)
        _call("grat_selected_attention_bwd", ctypes.byref(seq), *(ctypes.byref(_tensor(t)) for t in (dO, Q, K, V, O)), where,
              *(ctypes.byref(_tensor(t)) for t in (dQ, dK, dV)), float(scale), *lists, work.data_ptr() if work is not None else None, s,
              written=() if out is None else grads)
    return dQ, dK, dV
