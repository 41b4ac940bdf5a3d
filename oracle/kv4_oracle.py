"""The 4-bit K/V format and attention over it in 64 bits, with numpy only: a row of 128 values is four blocks of 32, a block is a
scale byte s (2^(s - 127); 255: not a number) and 32 codes into GRID with a sign."""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x: np.ndarray):
    """(codes uint8 [..., 128] of 0 .. 15, scale bytes uint8 [..., 4]) of rows [..., 128].  s puts the block's largest magnitude into
    [3.5, 7) units, but is at least 2; a value goes to the nearest grid point, halfway to the even code."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(*x.shape[:-1], 4, 32)
    with np.errstate(invalid="ignore"):
        amax = np.abs(blocks).max(-1)
    finite = np.isfinite(blocks).all(-1)
    m, e = np.frexp(np.where(finite, amax, 1.0))              # amax = m 2^e, 0.5 <= m < 1
    unit = np.maximum(e - 3 + (m >= 0.875), 2 - 127)
    unit = np.where(amax == 0, 2 - 127, unit)
    y = np.abs(np.where(finite[..., None], blocks, 0.0)) * np.exp2(-unit.astype(np.float64))[..., None]
    mids = (GRID[:-1] + GRID[1:]) / 2
    # a value on a midpoint goes to the even one of its neighbours: code i + 1 where i is odd
    code = np.zeros(y.shape, dtype=np.uint8)
    for i, mid in enumerate(mids):
        code += (y >= mid) if i % 2 else (y > mid)
    code |= (np.signbit(blocks).astype(np.uint8) << 3)
    code = np.where(finite[..., None], code, 0).astype(np.uint8)
    s = np.where(finite, unit + 127, 255).astype(np.uint8)
    return code.reshape(x.shape), s


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """Rows [..., 128] of codes [..., 128] and scale bytes [..., 4]."""
    g = np.concatenate([GRID, -GRID])[codes].reshape(*codes.shape[:-1], 4, 32)
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (g * s[..., None]).reshape(codes.shape)


def rows_of(codes: np.ndarray, scales: np.ndarray, pages, page_size: int, pos):
    """K and V (fp64 [n, 128] each) of positions `pos` of a sequence with the pool pages `pages`, for one KV head: codes uint8
    [n_pages, page_size, 128 bytes], scales uint8 [n_pages, page_size * 8]."""
    pos = np.asarray(pos, dtype=np.int64)
    page, slot = np.asarray(pages)[pos // page_size], pos % page_size
    byte = codes[page, slot]
    nib = np.stack([byte & 15, byte >> 4], axis=-1).reshape(len(pos), 256)
    sc = scales.reshape(scales.shape[0], page_size // 4, 2, 4, 4)[page, slot // 4, :, :, slot % 4]
    return values(nib[:, :128], sc[:, 0]), values(nib[:, 128:], sc[:, 1])


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float):
    """(out [128], lse, sum of p |v| [128], largest scale * sum |q_i k_i|) of one query over rows k, v."""
    if len(k) == 0:
        return np.zeros(128), -np.inf, np.zeros(128), 0.0
    x = (k @ q) * scale
    m = x.max()
    p = np.exp(x - m)
    return (p @ v) / p.sum(), m + np.log(p.sum()), (p @ np.abs(v)) / p.sum(), float((np.abs(k) @ np.abs(q)).max() * scale)


def local_positions(n: int, sink: int, window: int) -> np.ndarray:
    t = np.arange(n)
    return t[(t < sink) | (t > n - 1 - window)]
