"""The operators of include/qoda_matrices.h from their formulas, in numpy and 64 bits."""
from __future__ import annotations

import numpy as np

import operator_definitions as D

MX_KEY = 0x6D78666F75726269
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def mx_lots(rows, cols, seed, offset):
    return D.lots(rows, cols, seed ^ MX_KEY ^ D.KEY, offset)


def mx(x, stochastic=False, seed=0, offset=0):
    """(codes of every entry, exponents of every block; a block that is NaN has 128) of a matrix of fp32 or bf16 numbers, held in 64 bits."""
    rows, cols = x.shape
    blocks = -(-cols // 32)
    v = np.zeros((rows, blocks * 32))
    v[:, :cols] = x
    v = v.reshape(rows, blocks, 32)
    bad = ~np.isfinite(v).all(-1)
    w = np.where(bad[..., None], 0.0, v)
    most = np.abs(w).max(-1, initial=0.0)
    e = np.frexp(most)[1] - 3
    if stochastic:
        e = e + (most > 6 * np.exp2(e.astype(float)))
    e = np.where(most > 0, np.maximum(e, -127), -127)
    u = np.abs(w) / np.exp2(e.astype(float))[..., None]
    k = np.clip(np.searchsorted(GRID, u, side="right") - 1, 0, 6)
    low, high = GRID[k], GRID[k + 1]
    if stochastic:
        lots = mx_lots(rows, blocks * 32, seed, offset).reshape(rows, blocks, 32).astype(float)
        up = lots + 0.5 <= 65536 * (u - low) / (high - low)
    else:
        mid = (low + high) / 2
        up = (u > mid) | ((u == mid) & (k % 2 == 1))
    codes = k + up + 8 * np.signbit(w)
    codes = np.where(bad[..., None], 0, codes).reshape(rows, blocks * 32)
    codes[:, cols:] = 0
    return codes[:, :cols], np.where(bad, 128, e)


def mx_values(codes, e):
    rows, cols = codes.shape
    v = np.where(codes >= 8, -1.0, 1.0) * GRID[codes & 7]
    scale = np.where(e == 128, np.nan, np.exp2(e.astype(float)))
    return v * np.repeat(scale, 32, axis=1)[:, :cols]


def rounded(x, *args):
    return mx_values(*mx(x, *args))


def laid_out(codes, e):
    """(codes, scales) as they lie in memory."""
    rows, cols = codes.shape
    steps = -(-cols // 256)
    full = np.zeros((rows, steps * 256), dtype=np.uint8)
    full[:, :cols] = codes
    packed = full[:, 0::2] | full[:, 1::2] << 4
    groups = -(-rows // 64)
    scales = np.zeros((2 * steps, groups, 4, 4, 4, 2, 2), dtype=np.uint8)
    for block in range(e.shape[1]):
        r = np.arange(rows)
        scales[block // 4, r // 64, block % 4, r // 8 % 4, r % 4, r // 32 % 2, r // 4 % 2] = e[:, block] + 127
    return packed, scales.reshape(2 * steps, groups, 256)


def orthogonalize(g, steps, coefficients, eps):
    a, b, c = coefficients
    x = g / (np.sqrt((g * g).sum((-2, -1), keepdims=True)) + eps)
    for _ in range(steps):
        s = x @ np.swapaxes(x, -1, -2)
        x = a * x + (b * s + c * s @ s) @ x
    return x
