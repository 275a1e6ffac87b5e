"""Rotary positions in extended precision on the CPU, from the definitions: numpy, no code of the product."""
from __future__ import annotations

import math

import numpy as np
import torch

TURN = 2 * np.longdouble("3.14159265358979323846264338327950288")


def frequencies(rot_dim, theta, scaling="none", factor=1.0, low=1.0, high=32.0, original_len=0, divisors=None) -> np.ndarray:
    """f_i in radians per position."""
    r, L = rot_dim, np.longdouble
    theta, factor = L(theta), L(factor)
    if scaling == "base":
        theta = theta * factor ** (L(r) / (r - 2))
    f = np.array([theta ** (-L(2 * i) / r) for i in range(r // 2)])
    if scaling == "linear":
        return f / factor
    if scaling == "list":
        return f / np.array([L(v) for v in divisors])
    if scaling == "bands":
        n = original_len * f / TURN
        return np.where(n >= high, f, np.where(n <= low, f / factor,
                                               f * (n - low) / L(high - low) + f / factor * (high - n) / L(high - low)))
    if scaling == "ramp":
        at = lambda n: r * math.log(original_len / (2 * math.pi * n)) / (2 * math.log(float(theta)))
        a, b = max(math.floor(at(high)), 0), min(math.ceil(at(low)), r - 1)
        w = np.clip((np.arange(r // 2, dtype=L) - a) / L(max(b - a, 0.001)), 0, 1)
        return f * (1 - w) + f / factor * w
    return f


def turned(x: torch.Tensor, pos, f: np.ndarray, layout: str, rot_start: int, magnitude=1.0, transpose=False):
    """(y, far) as float64 ``[T, heads, d]``: the formula, and how far products in fp32 may be from it before the result is
    rounded.  cos and sin are off by 2^-22 at most: an angle held to 2^-32 turns (2^-29), its quadrant's rest rounded to
    fp32 (2^-26 radians), the function's own error of an ulp (2^-24) and the product with the magnitude (2^-24).  The two
    products and their sum are rounded to 2^-24 of themselves each: |error| <= 2^-21 magnitude (|u| + |v|)."""
    y = x.to(torch.float64).cpu().numpy().copy()
    far = np.zeros(y.shape)
    r, half = 2 * len(f), len(f)
    i = np.arange(half)
    u, v = (rot_start + i, rot_start + half + i) if layout == "half" else (rot_start + 2 * i, rot_start + 2 * i + 1)
    angle = np.asarray([int(p) for p in pos], np.longdouble)[:, None] * f
    angle = (angle - TURN * np.floor(angle / TURN)).astype(np.float64)[:, None, :]
    c, s = np.cos(angle) * magnitude, np.sin(angle) * magnitude * (-1 if transpose else 1)
    a, b = y[..., u].copy(), y[..., v].copy()
    y[..., u], y[..., v] = a * c - b * s, b * c + a * s
    far[..., u] = far[..., v] = 2.0 ** -21 * magnitude * (np.abs(a) + np.abs(b))
    assert r <= y.shape[-1]
    return y, far


def close(got: torch.Tensor, y: np.ndarray, far: np.ndarray) -> None:
    """Half a step of the type on top; where `far` is zero the values are the input's own."""
    g = got.to(torch.float64).cpu().numpy()
    info = torch.finfo(got.dtype)
    bound = np.where(far > 0, far + info.eps / 2 * (np.abs(y) + far) + info.smallest_normal * info.eps, 0.0)
    off = np.abs(g - y)
    assert (off <= bound).all(), (off - bound).max()


def to_bf16(y: np.ndarray) -> torch.Tensor:
    """Nearest bf16 of float64 values, ties to even, in one rounding (normal values)."""
    m, e = np.frexp(y)
    return torch.from_numpy(np.ldexp(np.round(m * 256.0), e - 8)).to(torch.float32).to(torch.bfloat16)
