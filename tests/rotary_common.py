"""Plain 64-bit reference of rotary positions, and a few things the tests around the attention share."""
from __future__ import annotations

import numpy as np
import torch

HALF, INTERLEAVED = 0, 1


def frequencies(rotary: int, base: float) -> np.ndarray:
    return base ** (-2.0 * np.arange(rotary // 2) / max(rotary, 1))


def rotate64(x: np.ndarray, pos, theta: np.ndarray, style: int, factor: float = 1.0) -> np.ndarray:
    """x float64 [n][heads][D], turned by pos [n]: the first 2 * len(theta) channels, the others as they are."""
    out, n = x.copy(), len(theta)
    a = np.asarray(pos, np.float64)[:, None] * theta[None, :]
    c, s = factor * np.cos(a)[:, None, :], factor * np.sin(a)[:, None, :]
    i = np.arange(n)
    i0, i1 = (i, i + n) if style == HALF else (2 * i, 2 * i + 1)
    out[..., i0] = x[..., i0] * c - x[..., i1] * s
    out[..., i1] = x[..., i0] * s + x[..., i1] * c
    return out


def rotation_tolerance(x: np.ndarray, theta: np.ndarray, style: int, factor: float, out_type) -> np.ndarray:
    """Bound on a rotated value formed in fp32 and rounded once: c and s, one product and the fused sum are each off by 2^-24 of
    factor * (|a| + |b|) at most, and half a step of the result's type."""
    n = len(theta)
    i = np.arange(n)
    i0, i1 = (i, i + n) if style == HALF else (2 * i, 2 * i + 1)
    big = np.zeros_like(x)
    big[..., i0] = big[..., i1] = abs(factor) * (np.abs(x[..., i0]) + np.abs(x[..., i1]))
    u = torch.finfo(out_type).eps / 2
    least = 2.0 ** -25 if out_type == torch.float16 else 1e-38
    rest = np.where(big > 0, u * big * 1.01 + 4 * 2.0 ** -24 * big + least, 0.0)      # channels that are not rotated: exact
    return rest
