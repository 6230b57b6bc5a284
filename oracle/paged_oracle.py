"""Oracle of the cache in pages: what it holds for given rows, and attention over it, in float64.

TEST INFRASTRUCTURE ONLY, like rkv_oracle: it shares no code with the library and imports nothing from the package.

Blocks of 32 channels share a power of two.  The grids are the OCP formats E4M3 (sign, 4 exponent bits with bias 7, 3 bits after
the point; the all-ones pattern is NaN, so 448 is the largest number) and E2M1 (0, 0.5, 1, 1.5, 2, 3, 4, 6).  The scale is the
smallest power of two that brings the block's largest magnitude to at most the format's largest number, but not below the one
whose smallest code is still a number of the cache's type.
"""
from __future__ import annotations

import numpy as np

BLOCK = 32
E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
E4M3 = np.array([i * 2.0**-9 if i < 8 else (8 + i % 8) * 2.0 ** (i // 8 - 10) for i in range(127)])


def limits(bits: int, dtype: str):
    """(grid, smallest exponent of a scale, largest magnitude that grid times power of two shares with the type)"""
    grid = E4M3 if bits == 8 else E2M1
    largest = {"fp16": 65504.0, "bf16": 2.0**128 - 2.0**120}[dtype]
    unit = {"fp16": -24, "bf16": -133}[dtype]                  # the type's smallest number is 2^unit
    low = unit + (9 if bits == 8 else 1)                       # 2^low times the grid's smallest step
    if dtype == "bf16":                                        # the scale's byte leaves room for 2^-126 at the least, and
        low = -118 if bits == 8 else -126                      # 2^-127 (a subnormal) is as small as the codes go
    exponent = {"fp16": 15, "bf16": 127}[dtype]
    top = (1.875 if bits == 8 else 1.5) * 2.0**exponent
    assert top <= largest
    return grid, low, top


def scales(x: np.ndarray, bits: int, dtype: str) -> np.ndarray:
    """Exponents of the blocks' scales (NaN where a block is not finite); x [..., channels] float64."""
    grid, low, _ = limits(bits, dtype)
    a = np.abs(x.reshape(*x.shape[:-1], x.shape[-1] // BLOCK, BLOCK)).max(-1)
    e = np.full(a.shape, float(low))
    for k in range(low, 128):                                  # by trying them all
        e = np.where(a > grid[-1] * 2.0**k, k + 1.0, e)
    return np.where(np.isfinite(a), e, np.nan)


def stored(x: np.ndarray, bits: int, dtype: str) -> np.ndarray:
    """The numbers that a cache holds for rows x [..., channels] (float64 values of the type)."""
    if bits == 16:
        return x.copy()
    grid, _, top = limits(bits, dtype)
    e = np.repeat(scales(x, bits, dtype), BLOCK, axis=-1).reshape(x.shape)
    two = np.exp2(np.where(np.isnan(e), 0, e))
    y = np.minimum(np.abs(np.where(np.isnan(e), 0, x)), top) / two
    hi = np.clip(np.searchsorted(grid, y), 1, len(grid) - 1)
    lo = hi - 1
    down, up = y - grid[lo], grid[hi] - y
    pick = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    return np.where(np.isnan(e), np.nan, np.sign(x) * grid[pick] * two)


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, first: int, causal=True, window=0, scale=None):
    """One sequence: q [n, Hq, D] at positions first .., k and v [L, Hkv, D] as stored -> out, lse, and what error bounds
    need: spread (sum of weight times |v|), reach (largest sum of |q||k| times the scale over the tokens a row sees) and mass
    (sum of their |v|)."""
    n, Hq, D = q.shape
    L, Hkv = k.shape[:2]
    scale = D**-0.5 if scale is None else scale
    p = np.arange(first, first + n)[:, None]
    t = np.arange(L)[None]
    sees = np.repeat(p >= 0, L, axis=1)                        # a row in front of the first token sees nothing
    if causal:
        sees &= t <= p
    if window:
        sees &= t > p - window
    out, spread, mass = (np.zeros((n, Hq, D)) for _ in range(3))
    lse, reach = np.full((n, Hq), -np.inf), np.zeros((n, Hq))
    for h in range(Hq):
        g = h // (Hq // Hkv)
        for i in range(n):
            vis = sees[i]
            if not vis.any():
                continue
            kk, vv = k[vis, g], v[vis, g]
            s = kk @ q[i, h] * scale
            m = s.max()
            if m == -np.inf:
                continue
            w = np.exp(s - m)
            lse[i, h] = m + np.log(w.sum())
            w /= w.sum()
            out[i, h], spread[i, h] = w @ vv, w @ np.abs(vv)
            mass[i, h] = np.abs(vv).sum(0)
            reach[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * abs(scale)
    return out, lse, spread, reach, mass
