"""What a 4-bit cache holds (fp64, CPU): groups of 32 values as small multiples of a shared
power of two.

A group's largest magnitude m gives the unit u = 2^max(floor(log2 m) - 2, -127).  Its
values are multiples of u / 2 below 2 u, of u below 4 u, of 2 u from there on, the
nearest one, of two the one that is an even number of these steps, and 6 u at most; a
group with an infinity or a NaN is NaN throughout.  Groups: 32 channels of a key, and 32
tokens of a channel of V within a page (fewer at its end).
"""
from __future__ import annotations

import numpy as np

GROUP = 32


def held(x: np.ndarray) -> np.ndarray:
    """The last axis is one group, of at most 32 values."""
    x = np.asarray(x, dtype=np.float64)
    assert x.shape[-1] <= GROUP
    m = np.abs(x).max(-1, keepdims=True)
    fine = np.isfinite(m)
    safe = np.where(fine & (m > 0), m, 1.0)
    u = np.exp2(np.maximum(np.floor(np.log2(safe)) - 2, -127.0))
    a = np.where(fine, np.abs(x), 0.0) / u
    step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
    y = np.minimum(np.rint(a / step) * step, 6.0) * u * np.sign(np.where(fine, x, 0.0))
    return np.where(fine, y, np.nan)


def held_keys(k: np.ndarray) -> np.ndarray:
    """[..., channel]"""
    g = k.reshape(k.shape[:-1] + (-1, GROUP))
    return held(g).reshape(k.shape)


def held_values(v: np.ndarray, tokens_per_page: int) -> np.ndarray:
    """[token, head, channel], the tokens of whole pages"""
    out = np.empty(v.shape, dtype=np.float64)
    for p in range(0, v.shape[0], tokens_per_page):
        for b in range(p, p + tokens_per_page, GROUP):
            e = min(b + GROUP, p + tokens_per_page)
            out[b:e] = np.moveaxis(held(np.moveaxis(v[b:e], 0, -1)), -1, 0)
    return out
