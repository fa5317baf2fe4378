"""float64 statement of the 4-bit format of the key/value cache (numpy; test infrastructure only).

A group of neighbouring values x is held as m = min x, a step s and codes c in 0 .. 15, and stands for m + s c:
s = fl(fl(max x - min x) fl(1 / 15)) rounded up to the 16-bit type, c = nearest integer (ties to even) of fl(x - m) fl(1 / s), fl = round to
fp32, the product exact.  s below 2^-126 is 0; a group with a NaN, an infinity or a range beyond 2^94 is NaN.
"""
from __future__ import annotations

import numpy as np


def _fl(x):
    with np.errstate(over="ignore", invalid="ignore"):
        return np.asarray(x, np.float64).astype(np.float32).astype(np.float64)


def _neighbours(x, dtype):
    """x >= 0 rounded down and up to the 16-bit type (float64)."""
    x = np.asarray(x, np.float64)
    lowest = -24 if dtype == "f16" else -133
    bits = 11 if dtype == "f16" else 8
    e = np.floor(np.log2(np.where(x > 0, x, 1.0)))
    step = 2.0 ** np.maximum(e - bits + 1, lowest)
    return np.floor(x / step) * step, np.ceil(x / step) * step


def round16(x, dtype):
    """x rounded to the nearest value of the 16-bit type, ties to even (finite results only; float64)."""
    x = np.asarray(x, np.float64)
    out = np.full(x.shape, np.nan)
    ok = np.isfinite(x)
    a = np.abs(x[ok])
    bits, lowest = (11, -24) if dtype == "f16" else (8, -133)
    e = np.floor(np.log2(np.where(a > 0, a, 1.0)))
    step = 2.0 ** np.maximum(e - bits + 1, lowest)
    out[ok] = np.copysign(np.round(a / step) * step, x[ok])      # np.round: ties to even
    return out


def quantise(x, group: int, dtype: str):
    """x [..., D] (values of the 16-bit type, float64) -> m, s [..., D] (spread over their groups), codes [..., D]."""
    x = np.asarray(x, np.float64)
    D = x.shape[-1]
    g = min(group, D)
    z = x.reshape(*x.shape[:-1], D // g, g)
    with np.errstate(over="ignore", invalid="ignore"):
        low, high = z.min(-1, keepdims=True), z.max(-1, keepdims=True)        # NaN propagates
        span = _fl(high - low)
        bad = ~(span <= 2.0 ** 94)
        span, low = np.where(bad, 0.0, span), np.where(bad, 0.0, low)
        s = _neighbours(_fl(span * float(np.float32(1.0 / 15.0))), dtype)[1]
        s = np.where(s < 2.0 ** -126, 0.0, s)
        inverse = np.where(s > 0, _fl(1.0 / np.where(s > 0, s, 1.0)), 0.0)
        c = np.round(_fl(np.where(bad, 0.0, z) - low) * inverse)
    assert c.min(initial=0) >= 0 and c.max(initial=0) <= 15
    spread = lambda a: np.broadcast_to(np.where(bad, np.nan, a), z.shape).reshape(x.shape)  # noqa: E731
    return spread(low), spread(s), c.reshape(x.shape)


def read_back(m, s, c, dtype: str):
    """What comes back in 16 bits: m + s c in fp32, rounded once more; the largest number where f16 ends (s is rounded up)."""
    x = round16(_fl(m + s * c), dtype)
    return np.where(x > 65504.0, 65504.0, x) if dtype == "f16" else x
