"""Float64 CPU oracle of the operators that train a network around the filter -- TEST INFRASTRUCTURE ONLY.

    out = drop(act(x w + b)) + residual and its gradients; LayerNorm of a residual sum and its gradients;
    dropout from a counter-based generator.

drop() keeps element e (its flat index) where number e % 8 of group e // 8 is at least T = 65536 p rounded,
and scales by 65536 / (65536 - T).  The numbers are the 16-bit halves, low ones first, of the words of
Philox4x32 with seven rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3",
2011) of the counter (group low, group high, place low, place high) under the seed.
"""
from __future__ import annotations

import numpy as np
from scipy.special import erf, ndtr

LOW = np.uint64(0xFFFFFFFF)
HALF = np.uint64(32)


def philox4x32(counter, key, rounds: int):
    """Four words of 32 bits (as uint64 arrays) from four counter words and two key words."""
    c = [np.asarray(v, dtype=np.uint64) for v in counter]
    k = [int(v) for v in key]
    for _ in range(rounds):
        p = c[0] * np.uint64(0xD2511F53)
        q = c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> HALF) ^ c[1] ^ np.uint64(k[0]), q & LOW, (p >> HALF) ^ c[3] ^ np.uint64(k[1]), p & LOW]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def threshold(p: float) -> int:
    return int(np.rint(np.float64(np.float32(p)) * 65536.0))


def keep(n: int, p: float, seed: int, offset: int = 0, counter: int = 0) -> np.ndarray:
    """Which of n elements are kept."""
    T = threshold(p)
    if T == 0:
        return np.ones(n, dtype=bool)
    place = (offset + counter) % 2 ** 64
    i = np.arange((n + 7) // 8, dtype=np.uint64)
    full = lambda v: np.full(i.shape, v, dtype=np.uint64)  # noqa: E731
    words = philox4x32((i & LOW, i >> HALF, full(place & 0xFFFFFFFF), full(place >> 32)),
                       (seed & 0xFFFFFFFF, seed >> 32), 7)
    numbers = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=-1)
    return numbers.reshape(-1)[:n] >= T


def drop(y: np.ndarray, p: float = 0.0, seed: int = 0, offset: int = 0, counter: int = 0) -> np.ndarray:
    T = threshold(p)
    k = keep(y.size, p, seed, offset, counter).reshape(y.shape)
    return np.where(k, y * (65536.0 / (65536 - T)), 0.0)


def act(z, name: str):
    if name == "relu":
        return np.where(z < 0, 0.0, z)
    return z * ndtr(z) if name == "gelu" else z


def act_slope(z, name: str):
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "gelu":
        return 0.5 * (1.0 + erf(z / np.sqrt(2.0))) + z * np.exp(-0.5 * z * z) / np.sqrt(2.0 * np.pi)
    return np.ones_like(z)


def linear(x, w, b=None, activation="none", residual=None, **rng):
    """out and the value before the activation."""
    z = x @ w + (0.0 if b is None else b)
    out = drop(act(z, activation), **rng)
    return out + (0.0 if residual is None else residual), z


def linear_backward(g, x, w, pre=None, activation="none", **rng):
    """dx, dw, db and dz."""
    dz = drop(g, **rng)
    if activation == "relu":  # a unit that is off passes on 0, whatever reaches it
        dz = np.where(pre > 0, dz, 0.0)
    elif activation != "none":
        dz = dz * act_slope(pre, activation)
    return dz @ w.T, x.T @ dz, dz.sum(0), dz


def layer_norm(v, gamma, beta, eps):
    mean = v.mean(-1, keepdims=True)
    return (v - mean) / np.sqrt(((v - mean) ** 2).mean(-1, keepdims=True) + eps) * gamma + beta


def layer_norm_backward(g, v, gamma, eps, gsum=None):
    """dx, dgamma, dbeta."""
    mean = v.mean(-1, keepdims=True)
    sd = np.sqrt(((v - mean) ** 2).mean(-1, keepdims=True) + eps)
    h, a = (v - mean) / sd, g * gamma
    dx = (a - a.mean(-1, keepdims=True) - h * (a * h).mean(-1, keepdims=True)) / sd
    return dx + (0.0 if gsum is None else gsum), (g * h).sum(0), g.sum(0)
