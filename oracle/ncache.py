"""Float64 oracle of the 4-bit cache: rows of e2m1 codes, one power-of-two scale for every 32 channels."""
from __future__ import annotations

import math

import numpy as np

NGROUP = 32
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
LEAST_EXPONENT, MOST_EXPONENT = -100, 125


def n_round(y: np.ndarray) -> np.ndarray:
    """y rounded to the nearest e2m1 value, ties to the even code; magnitudes above 6 to 6."""
    y = np.asarray(y, np.float64)
    _, e = np.frexp(y)                                   # |y| = m 2^e, 0.5 <= m < 1
    step = np.ldexp(1.0, np.maximum(e - 1, 0) - 1)       # one mantissa bit; subnormals below 1
    return np.copysign(np.minimum(np.abs(np.rint(y / step) * step), 6.0), y)


def n_scale(amax: float) -> float:
    """The smallest power of two (exponents LEAST to MOST) with amax <= 6 * scale; NaN if amax is not finite."""
    if not math.isfinite(amax):
        return math.nan
    e = LEAST_EXPONENT
    while e < MOST_EXPONENT and math.ldexp(6.0, e) < amax:
        e += 1
    return math.ldexp(1.0, e)


def n_rows(x: np.ndarray):
    """Codes (as numbers) and scales of rows x [m][d]: codes [m][d], scales [m][d / 32]."""
    x = np.asarray(x, np.float64)
    g = x.reshape(len(x), -1, NGROUP)
    amax = np.where(np.isfinite(g).all(axis=2), np.abs(np.where(np.isfinite(g), g, 0)).max(axis=2), math.inf)
    scales = np.vectorize(n_scale, otypes=[np.float64])(amax)
    with np.errstate(invalid="ignore"):
        codes = n_round(np.where(np.isnan(scales)[..., None], 0.0, g / scales[..., None]))
    return codes.reshape(x.shape), scales


def n_values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    return codes * np.repeat(scales, NGROUP, axis=-1)


def n_bytes(codes: np.ndarray, scales: np.ndarray):
    """As the cache holds them: packed codes [m][d / 2] and scale bytes [m][d / 32], uint8."""
    c = np.searchsorted(MAGNITUDES, np.abs(codes)) + 8 * np.signbit(codes)
    bad = np.isnan(scales)
    e = np.frexp(np.where(bad, 1.0, scales))[1] - 1
    return (c[:, 0::2] + 16 * c[:, 1::2]).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def n_unpack(packed: np.ndarray, scale_bytes: np.ndarray) -> np.ndarray:
    """Stored values of rows as the cache holds them."""
    table = np.array(MAGNITUDES + tuple(-m for m in MAGNITUDES))
    codes = np.stack([table[packed & 15], table[packed >> 4]], axis=-1).reshape(*packed.shape[:-1], 2 * packed.shape[-1])
    s = np.where(scale_bytes == 255, math.nan, np.ldexp(1.0, scale_bytes.astype(np.int64) - 127))
    return n_values(codes, s)
