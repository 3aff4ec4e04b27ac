"""The operators on 8-bit prefix records in 64 bits, straight from their definitions (numpy, one environment at a time)."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 32
# the value of every e4m3 code (0x7f and 0xff are NaN)
VALUES = np.array([(-1.0 if c & 128 else 1.0) * (math.nan if c & 127 == 127 else ((c & 7) * 2.0 ** -9 if c & 120 == 0 else
                  (1 + (c & 7) / 8) * 2.0 ** (((c >> 3) & 15) - 7))) for c in range(256)])


def block_scale(amax: float) -> float:
    if amax == 0.0:
        return 1.0
    s = 2.0 ** max(-126, math.floor(math.log2(amax)) - 10)
    while amax / s > 448.0:
        s *= 2.0
    return s


def encode(x: np.ndarray) -> np.ndarray:
    """Codes of x (already divided by the scale): nearest value, ties to the even code, saturated, NaN -> 0x7f."""
    a = np.minimum(np.abs(x), 448.0)
    grid = VALUES[:127]
    hi = np.clip(np.searchsorted(grid, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - a, a - grid[lo]
    k = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    k = np.where(np.isnan(x), 127, k | np.where(np.signbit(x), 128, 0))
    return k.astype(np.uint8)


def quantize_head(x: np.ndarray, visible: np.ndarray):
    """x [len, hd] of one head and plane -> (codes, scales of its blocks; a block with a NaN has a minus)."""
    codes, scales = np.zeros(x.shape, np.uint8), []
    for b in range(0, len(x), BLOCK):
        blk = np.where(visible[b:b + BLOCK, None], x[b:b + BLOCK], 0.0)
        fin = np.abs(blk[np.isfinite(blk)])
        s = block_scale(float(fin.max()) if fin.size else 0.0)
        codes[b:b + BLOCK] = encode(blk / s)
        scales.append(-s if np.isnan(blk).any() else s)
    return codes, np.array(scales)


def scores(q, k, scale):
    """q [rows, hd], k [tokens, hd] -> (scale q k^T, and the same of the absolute values: what rounding errors go by)."""
    return scale * (q @ k.T), abs(scale) * (np.abs(q) @ np.abs(k).T)


def attend(q, k, v, scale):
    """(out, lse, the largest absolute-value score) for rows of q against the visible tokens' keys and values."""
    if len(k) == 0:
        return np.zeros((len(q), v.shape[-1])), np.full(len(q), -np.inf), 0.0
    s, sa = scores(q, k, scale)
    m = s.max(1, keepdims=True)
    p = np.exp(s - m)
    z = p.sum(1, keepdims=True)
    return (p / z) @ v, (m + np.log(z))[:, 0], float(sa.max())


def weigh(q, lse, k, scale):
    s, sa = scores(q, k, scale)
    with np.errstate(invalid="ignore"):
        return np.where(np.isfinite(lse)[:, None], np.exp(s - lse[:, None]), 0.0).sum(0), float(sa.max()) if sa.size else 0.0


def select(weight, visible, n, keep, first, last):
    """Ascending indices of the kept tokens."""
    def key(t):
        if t < first or t >= n - last:
            return math.inf
        w = float(weight[t])
        return -math.inf if math.isnan(w) or not visible[t] else w
    return sorted(sorted(range(n), key=lambda t: (-key(t), t))[:min(keep, n)])
