"""Float64 oracle of rotary positions."""
from __future__ import annotations

import numpy as np


def frequencies(d_rot: int, base: float = 10000.0, mode: str = "none", stretch: float = 1.0, length: float = 0.0,
                few: float = 1.0, many: float = 32.0) -> np.ndarray:
    i = np.arange(d_rot // 2, dtype=np.float64)
    if mode == "base":
        base = base * stretch ** (d_rot / (d_rot - 2))
    f = base ** (-2 * i / d_rot)
    if mode in ("none", "base"):
        return f
    if mode == "linear":
        return f / stretch
    if mode == "turns":
        g = np.clip((length * f / (2 * np.pi) - few) / (many - few), 0, 1)
    else:
        c = lambda r: d_rot * np.log(length / (2 * np.pi * r)) / (2 * np.log(base))
        lo, hi = np.clip(np.floor(c(many)), 0, d_rot - 1), np.clip(np.ceil(c(few)), 0, d_rot - 1)
        g = 1 - np.clip((i - lo) / (hi - lo if hi != lo else 0.001), 0, 1)
    return g * f + (1 - g) * f / stretch


def rotary(x, positions, freq, interleaved: bool = False, transpose: bool = False, factor: float = 1.0) -> np.ndarray:
    """x [N][heads][d] turned by positions [N] times freq [d_rot / 2]."""
    x = np.asarray(x, np.float64)
    h = len(freq)
    a = np.asarray(positions, np.float64)[:, None, None] * np.asarray(freq, np.float64)
    c, s = np.cos(a) * factor, np.sin(a) * factor * (-1 if transpose else 1)
    y = x.copy()
    u, v = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if interleaved else (slice(0, h), slice(h, 2 * h))
    y[..., u] = x[..., u] * c - x[..., v] * s
    y[..., v] = x[..., u] * s + x[..., v] * c
    return y
