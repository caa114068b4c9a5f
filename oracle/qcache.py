"""Float64 oracle of the 8-bit cache: blocks of 64 rows, one power-of-two scale each for keys and for values."""
from __future__ import annotations

import math

import numpy as np

QBLOCK = 64
LARGEST = {"e4m3": 448.0, "int8": 127.0}
LEAST_EXPONENT = -100


def q_round(y: np.ndarray, fmt: str) -> np.ndarray:
    """y (within the codes' range) rounded to the nearest code, ties to even."""
    y = np.asarray(y, np.float64)
    if fmt == "int8":
        return np.rint(y)
    _, e = np.frexp(y)                                   # |y| = m 2^e, 0.5 <= m < 1
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)      # 3 mantissa bits; subnormals below 2^-6
    return np.rint(y / step) * step


def q_scale(amax: float, fmt: str) -> float:
    """The smallest power of two (exponent >= LEAST_EXPONENT) with amax <= LARGEST * scale; NaN if amax is not finite."""
    if not math.isfinite(amax):
        return math.nan
    e = LEAST_EXPONENT
    while math.ldexp(LARGEST[fmt], e) < amax:
        e += 1
    return math.ldexp(1.0, e)


def q_write(codes, scales, rows, start: int, fmt: str, bounds=None) -> None:
    """One pair, in place: rows [m][d] to codes [R][d] from row `start` on (rows past R are dropped)."""
    R = codes.shape[0]
    end = min(start + len(rows), R)
    if end <= start:
        return
    for b in range(start // QBLOCK, -(-end // QBLOCK)):
        lo, hi = b * QBLOCK, min((b + 1) * QBLOCK, end)
        first_new = max(lo, start)
        x = np.asarray(rows[first_new - start:hi - start], np.float64)
        if first_new > lo:
            x = np.concatenate([codes[lo:first_new] * scales[b], x])
        scales[b] = q_scale(float(np.abs(x).max()) if np.isfinite(x).all() else math.inf, fmt)
        codes[lo:hi] = q_round(x / scales[b], fmt) if math.isfinite(scales[b]) else 0.0
        if bounds is not None:
            bounds[b, 0], bounds[b, 1] = codes[lo:hi].min(axis=0), codes[lo:hi].max(axis=0)


def q_values(codes, scales) -> np.ndarray:
    """Stored values of one pair."""
    return np.asarray(codes, np.float64) * np.repeat(np.asarray(scales, np.float64), QBLOCK)[:len(codes), None]


def q_block_scores(Q, bounds, scales, length: int, scale: float, beta=None) -> np.ndarray:
    """One pair: Q [G][d], bounds [blocks][2][d] (codes), scales [blocks]."""
    Q = np.asarray(Q, np.float64)
    out = np.full(len(scales), -math.inf)
    for b in range(min(len(scales), -(-length // QBLOCK))):
        lo, hi = np.asarray(bounds[b], np.float64) * float(scales[b])
        out[b] = scale * np.maximum(Q * lo, Q * hi).sum(axis=1).max()
        if beta is not None:
            out[b] += np.asarray(beta[b * QBLOCK:min((b + 1) * QBLOCK, length)], np.float64).max()
    return out


def q_attend(Q, K, V, beta, K_f, V_f, scale: float):
    """One pair over the given rows: rows with beta = -inf are left out, no row gives zeros.  Returns (out, mass_abs):
    the output and sum_j p_j |v_j|, which a rounding error of the probabilities multiplies."""
    Q = np.asarray(Q, np.float64)
    keep = np.ones(len(K), bool) if beta is None else np.asarray(beta) > -math.inf
    K, V = np.asarray(K, np.float64)[keep], np.asarray(V, np.float64)[keep]
    b = np.zeros(len(K)) if beta is None else np.asarray(beta, np.float64)[keep]
    if K_f is not None:
        K, V = np.concatenate([K, np.asarray(K_f, np.float64)]), np.concatenate([V, np.asarray(V_f, np.float64)])
        b = np.concatenate([b, np.zeros(len(K_f))])
    if len(K) == 0:
        return np.zeros((len(Q), V.shape[1])), np.zeros((len(Q), V.shape[1]))
    X = scale * (Q @ K.T) + b
    E = np.exp(X - X.max(axis=1, keepdims=True))
    P = E / E.sum(axis=1, keepdims=True)
    return P @ V, P @ np.abs(V)
