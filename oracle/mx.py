"""TEST INFRASTRUCTURE ONLY: plain fp64 reference of the microscaled formats, the RMS norm and the 8-bit GQA cache.

Nothing in the product path imports this module; it shares no code with the HIP kernels.

Formats: a block shares a scale 2^(b - 127), b a byte, 1 <= b <= 254 (255: the block is NaN); entries under it are E4M3 (1 sign, 4 exponent,
3 mantissa bits, bias 7, largest 448, no infinities) or E2M1 (1, 2, 1 bits, bias 1: 0, .5, 1, 1.5, 2, 3, 4, 6).  b is the smallest with
which the block's largest finite magnitude does not pass the format's largest value; entries are rounded to nearest, halfway to the
even code.

RMS norm: h = bf16(x + residual), y = h w / sqrt(mean h^2 + eps).

8-bit GQA cache: a block is 16 consecutive positions of one KV head, keys and values each.  Writing rows p .. p + n - 1 into a block: with
p % 16 == 0 the block begins anew; otherwise its rows ahead of p stay, and the scale is the larger of the block's and the one the new rows
need; all values are rounded to that scale.  Rows behind the written ones are gone.
"""
from __future__ import annotations

import numpy as np

E4M3 = np.array([(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])
E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6.0])


def to_bf16(x):
    """nearest bf16 value (even), as fp64; x fp64 or fp32, finite"""
    x = np.asarray(x, dtype=np.float64)
    m, e = np.frexp(x)
    step = np.exp2(np.maximum(e - 8, -133).astype(np.float64))
    return np.rint(x / step) * step


def nearest(x, grid):
    """x rounded to +- the values of `grid` (increasing, from 0; magnitudes up to its last), halfway to the even index"""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x)
    assert (a <= grid[-1]).all()
    hi = np.clip(np.searchsorted(grid, a, side="left"), 0, len(grid) - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - a, a - grid[lo]
    return np.copysign(np.where((down < up) | ((down == up) & (lo % 2 == 0)), grid[lo], grid[hi]), x)


def scale_byte(amax, grid):
    """the smallest b >= 1 with amax <= grid[-1] 2^(b - 127)"""
    amax = np.asarray(amax, dtype=np.float64)
    _, e = np.frexp(amax)
    b = np.maximum(e + 127 - 12, 1)
    for _ in range(16):
        b = np.where(amax > grid[-1] * np.exp2(b - 127.0), b + 1, b)
    return np.where(amax == 0, 1, b).astype(np.int64)


def quantise(x, grid, block=32):
    """x [.., n]: (values, bytes [.., n / block])"""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(x.shape[:-1] + (-1, block))
    b = scale_byte(np.abs(blocks).max(-1), grid)
    s = np.exp2(b - 127.0)[..., None]
    return (nearest(blocks / s, grid) * s).reshape(x.shape), b


def rmsnorm(x, residual, weight, eps):
    """(y, h), y not rounded"""
    h = to_bf16(np.asarray(x, np.float64) + (0 if residual is None else np.asarray(residual, np.float64)))
    return h * np.asarray(weight, np.float64) / np.sqrt((h * h).mean(-1, keepdims=True) + eps), h


class Cache8:
    """One request's rows in the 8-bit cache: the values [n, heads, dim] they stand for, after writes in order."""

    def __init__(self, heads: int, dim: int):
        self.rows = np.zeros((0, heads, dim))
        self.b = np.zeros((0, heads), dtype=np.int64)

    def write(self, start: int, rows):
        rows = np.asarray(rows, dtype=np.float64)
        assert start <= len(self.rows)
        at, blocks, scales = 0, [], []
        while at < len(rows):
            blk, t = (start + at) // 16, (start + at) % 16
            n = min(16 - t, len(rows) - at)
            new = rows[at:at + n]
            b = scale_byte(np.abs(new).max((0, 2)), E4M3)
            kept = self.rows[blk * 16:blk * 16 + t]
            if t:
                b = np.maximum(b, self.b[blk])
            s = np.exp2(b - 127.0)[None, :, None]
            block = nearest(np.concatenate([kept, new]) / s, E4M3) * s
            blocks.append(block)
            scales.append(b)
            at += n
        if blocks:
            self.rows = np.concatenate([self.rows[:start - start % 16], *blocks])
            self.b = np.concatenate([self.b[:start // 16], np.stack(scales)])
