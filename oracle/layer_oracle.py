"""What a layer does around its product, in fp64 (numpy): bias, activation, dropout from a
counter-based generator, residual, and the gradient behind them, from the definitions in
include/lbp.h.  Shares no code with the CUDA path.

Philox4x32: Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3",
SC 2011.
"""
from __future__ import annotations

import numpy as np
from scipy.special import erfc

_M = (0xD2511F53, 0xCD9E8D57)
_W = (0x9E3779B9, 0xBB67AE85)
_LOW = np.uint64(0xFFFFFFFF)


def philox4x32(counter, key, rounds: int = 10):
    """counter: four uint32 arrays (or ints), key: two ints.  Four uint64 arrays of 32-bit words."""
    c = [np.asarray(v, dtype=np.uint64) for v in counter]
    k = [int(v) for v in key]
    for _ in range(rounds):
        a, b = c[0] * np.uint64(_M[0]), c[2] * np.uint64(_M[1])
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & _LOW,
             (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & _LOW]
        k = [(k[0] + _W[0]) & 0xFFFFFFFF, (k[1] + _W[1]) & 0xFFFFFFFF]
    return c


def numbers(n, seed: int, offset: int) -> np.ndarray:
    """u(n) for an array of element numbers."""
    n = np.asarray(n, dtype=np.uint64)
    group = n >> np.uint64(3)
    hi = ((offset >> 32) + (1 << 31)) & 0xFFFFFFFF
    words = philox4x32((group & _LOW, group >> np.uint64(32), np.full_like(group, offset & 0xFFFFFFFF),
                        np.full_like(group, hi)), (seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF))
    word = np.choose(((n & np.uint64(7)) >> np.uint64(1)).astype(np.int64), words)
    return (word >> ((n & np.uint64(1)) * np.uint64(16))) & np.uint64(0xFFFF)


def threshold(p: float) -> int:
    return int(np.floor(float(np.float32(p)) * 65536.0 + 0.5))


def keep(n, p: float, seed: int, offset: int) -> np.ndarray:
    return numbers(n, seed, offset) >= threshold(p)


def drop(v: np.ndarray, n, p: float, seed: int, offset: int) -> np.ndarray:
    t = threshold(p)
    if t == 0:
        return v
    scale = 65536.0 / (65536 - t) if t < 65536 else 0.0
    with np.errstate(invalid="ignore"):
        return np.where(keep(n, p, seed, offset), v * scale, 0.0)


def row_numbers(rows: int, C: int, first: int = 0, step: int = 0) -> np.ndarray:
    return first + np.arange(rows)[:, None] * (step or C) + np.arange(C)[None, :]


def act(z: np.ndarray, a: str) -> np.ndarray:
    if a == "relu":
        return np.where(z > 0, z, 0.0)
    if a == "gelu":
        return 0.5 * z * erfc(-z / np.sqrt(2.0))
    if a == "gelu_tanh":
        return 0.5 * z * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (z + 0.044715 * z ** 3)))
    if a == "silu":
        return z / (1.0 + np.exp(-z))
    return z


def act_slope(z: np.ndarray, a: str) -> np.ndarray:
    if a == "relu":
        return (z > 0).astype(np.float64)
    if a == "gelu":
        return 0.5 * erfc(-z / np.sqrt(2.0)) + z * np.exp(-0.5 * z * z) / np.sqrt(2.0 * np.pi)
    if a == "gelu_tanh":
        c = np.sqrt(2.0 / np.pi)
        t = np.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    if a == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return np.ones_like(z)
