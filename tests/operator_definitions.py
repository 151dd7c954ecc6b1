"""The operators of include/qoda_operators.h from their formulas, in numpy and 64 bits, and how far fp32 sums and a rounded store may be from them."""
from __future__ import annotations

import math

import numpy as np

KEY = 0x64726F706F757473
U32 = 2.0 ** -24          # half a unit of fp32
STORE = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}      # half a unit of 24 and of 8 significant bits

_erf = np.vectorize(math.erf, otypes=[np.float64])
_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def philox(c, k, rounds=10):
    """Philox4x32 on arrays of counters c[0..3] (uint64 holding 32 bits) and a key of two words."""
    m = np.uint64(0xFFFFFFFF)
    c = [np.asarray(v, dtype=np.uint64) & m for v in c]
    k0, k1 = int(k[0]), int(k[1])
    for _ in range(rounds):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), p1 & m, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p0 & m]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def lots(rows, cols, seed, offset, first_row=0):
    key = (seed ^ KEY) & (2**64 - 1)
    blocks = (cols + 7) // 8
    c0 = np.broadcast_to(np.arange(blocks, dtype=np.uint64)[None, :], (rows, blocks))
    c1 = np.broadcast_to((first_row + np.arange(rows, dtype=np.uint64))[:, None], (rows, blocks))
    full = lambda v: np.full((rows, blocks), v, dtype=np.uint64)  # noqa: E731
    w = philox([c0, c1, full(offset & 0xFFFFFFFF), full(offset >> 32)], (key & 0xFFFFFFFF, key >> 32))
    out = np.empty((rows, blocks, 8), dtype=np.uint64)
    for j in range(8):
        out[:, :, j] = w[j & 3] & np.uint64(0xFFFF) if j < 4 else w[j & 3] >> np.uint64(16)
    return out.reshape(rows, blocks * 8)[:, :cols]


def threshold(p):
    return int(math.floor(p * 65536 + 0.5))


def drop(v, p, seed, offset, first_row=0):
    t = threshold(p)
    if t == 0:
        return v
    kept = lots(v.shape[0], v.shape[1], seed, offset, first_row) >= t
    with np.errstate(invalid="ignore"):
        return np.where(kept, v * (65536.0 / (65536 - t) if t < 65536 else 0.0), 0.0)


def act(z, a):
    with np.errstate(all="ignore"):
        return {"none": lambda: z, "relu": lambda: np.where(z < 0, 0.0, z), "leaky_relu": lambda: np.where(z > 0, z, 0.2 * z),
                "gelu": lambda: z * 0.5 * _erfc(-z / math.sqrt(2)), "silu": lambda: z / (1 + np.exp(-z))}[a]()


def slope(z, a):
    with np.errstate(all="ignore"):
        s = 1 / (1 + np.exp(-z))
        return {"none": lambda: np.ones_like(z), "relu": lambda: (z > 0) * 1.0, "leaky_relu": lambda: np.where(z > 0, 1.0, 0.2),
                "gelu": lambda: 0.5 * _erfc(-z / math.sqrt(2)) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi),
                "silu": lambda: s * (1 + z * (1 - s))}[a]()


def linear(x, w, b=None, residual=None, a="none", p=0.0, seed=0, offset=0):
    z = x @ w.T + (0.0 if b is None else b)
    y = drop(act(z, a), p, seed, offset)
    return (y if residual is None else residual + y), z


def linear_input_grad(dz, w, pre=None, a="none", p=0.0, seed=0, offset=0, residual=None):
    dx = dz @ w
    dx = drop(dx if pre is None else dx * slope(pre, a), p, seed, offset)
    return dx if residual is None else residual + dx


def group_norm(x, groups, w, b, eps, a):
    n, s, c = x.shape
    v = x.reshape(n, s, groups, c // groups)
    mean = v.mean(axis=(1, 3))
    var = ((v - mean[:, None, :, None]) ** 2).mean(axis=(1, 3))
    rstd = 1 / np.sqrt(var + eps)
    h = ((v - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(n, s, c)
    z = h * w + b
    return act(z, a), mean, rstd, h, z


def group_norm_grad(dy, x, mean, rstd, groups, w, b, a):
    n, s, c = x.shape
    four = lambda t: t.reshape(n, s, groups, c // groups)  # noqa: E731
    h = (four(x) - mean[:, None, :, None]) * rstd[:, None, :, None]
    dh = dy * slope(h.reshape(n, s, c) * w + b, a)
    u = four(dh * w)
    dx = (u - u.mean(axis=(1, 3), keepdims=True) - h * (u * h).mean(axis=(1, 3), keepdims=True)) * rstd[:, None, :, None]
    return dx.reshape(n, s, c), (dh * h.reshape(n, s, c)).sum((0, 1)), dh.sum((0, 1)), u.reshape(n, s, c)


# ---- how far off: first-order bounds of fp32 sums of k terms in any order, with the activation's error and the store's rounding

ACT_ERROR = 6e-7           # of an activation's value and slope over 1 + |z|: the normal tail's formula is good to 1.5e-7, the rest is rounding


def sum_bound(k, magnitude):
    """A sum of k fp32 products whose magnitudes add up to ``magnitude``."""
    return (k + 4) * 2 * U32 * magnitude


def stored(bound, value, dtype):
    """``bound`` before the store, and the store's rounding of value (which may itself be off by the bound)."""
    return bound + (np.abs(value) + bound) * STORE[dtype] * 1.001 + 1e-38
