"""Helpers for the token-sequence tests: seeded tensors of every layout."""
import numpy as np
import torch

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# rounding to nearest: at most 2^-p relative with p significant bits, and half the smallest subnormal
ROUND = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
TINY = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25, "f32": 2.0 ** -150}


def normal(shape, dtype, seed, layout="heads", gain=1.0, device="cuda"):
    """[B, H, N, d] of N(0, gain^2): "heads" contiguous, "tokens" a view of [B, N, H, d], "wide" rows longer than d."""
    B, H, N, d = shape
    gen = torch.Generator().manual_seed(seed)
    x = (gain * torch.randn(shape, generator=gen)).to(TYPES[dtype])
    if layout == "tokens":
        x = x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    elif layout == "wide":
        buf = torch.full((B, H + 1, N + 2, d + 32), float("nan"), dtype=x.dtype)
        buf[:, :H, 1:N + 1, 16:16 + d] = x
        return buf.to(device)[:, :H, 1:N + 1, 16:16 + d]
    return x.to(device) if layout != "tokens" else x.permute(0, 2, 1, 3).contiguous().to(device).permute(0, 2, 1, 3)


def f64(t):
    return t.detach().double().cpu().numpy()


def ints(values, device="cuda"):
    return None if values is None else torch.tensor(values, dtype=torch.int32, device=device)


def nan_like(t):
    """An output in which every element that a kernel fails to store stays visible (same strides)."""
    return torch.empty_like(t).fill_(float("nan"))


def assert_rel(got, want, bound, what):
    """2-norm of the difference over that of the result."""
    assert np.isfinite(got).all(), f"{what}: not finite"
    off = np.linalg.norm(got - want)
    norm = np.linalg.norm(want)
    assert off <= bound * norm + 1e-300, f"{what}: relative error {off / max(norm, 1e-300):.3e}, bound {bound:.1e}"
