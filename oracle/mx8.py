"""Float64 CPU oracle of the operators in eight bits and of the root-mean-square norm -- TEST INFRASTRUCTURE ONLY.

Eight bits: rows in blocks of 32 channels, zeros behind the last channel; of a block the smallest s with which no finite
value is above 448 2^s, kept in -117 .. 119, and of a value the E4M3 number nearest to v / 2^s, ties to the even
code, at most 448 in size; NaN of a NaN or an infinity.
"""
from __future__ import annotations

import numpy as np

BLOCK = 32
#: the value of each code 0 .. 0x7e
CODES = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127])


def blocks(C: int) -> int:
    return -(-C // BLOCK)


def pack(v: np.ndarray):
    """Codes [M, 32 blocks] and scale bytes [M, blocks] of v [M, C]."""
    M, C = v.shape
    b = np.zeros((M, blocks(C), BLOCK))
    b.reshape(M, -1)[:, :C] = v
    top = np.where(np.isfinite(b), np.abs(b), 0.0).max(-1)
    s = np.full(top.shape, -117)
    for up in range(-117, 119):  # one more while the block does not fit
        s += (s == up) & (top > 448.0 * 2.0 ** up)
    u = np.abs(b) / 2.0 ** s[..., None]
    with np.errstate(invalid="ignore"):
        u = np.minimum(u, 448.0)
    at = np.searchsorted(CODES, np.where(np.isnan(u), 0.0, u), side="right") - 1  # the code at or below
    above = np.minimum(at + 1, 126)
    mid = (CODES[at] + CODES[above]) / 2
    at = np.where((u > mid) | ((u == mid) & (at % 2 == 1)), above, at)
    at = np.where(np.isfinite(b), at, 0x7F)
    code = at + 128 * np.signbit(b)
    return code.reshape(M, -1).astype(np.uint8), (s + 127).astype(np.uint8)


def unpack(code: np.ndarray, scale: np.ndarray, C: int) -> np.ndarray:
    low = (code & 127).astype(np.int64)
    v = np.where(low == 127, np.nan, CODES[np.minimum(low, 126)]) * np.where(code & 128, -1.0, 1.0)
    s = scale.astype(np.float64) - 127
    return (v.reshape(*scale.shape, BLOCK) * 2.0 ** s[..., None]).reshape(code.shape)[:, :C]


def half_step(size: np.ndarray) -> np.ndarray:
    """How far a rounded value of rows whose sizes are at most `size` [M, C] may be from its own."""
    M, C = size.shape
    code, scale = pack(size)
    s = np.repeat(scale.astype(np.float64) - 127, BLOCK, -1)[:, :C]
    return np.maximum(size * 2.0 ** -4, 2.0 ** (s - 10))


def rms_norm(v, gamma, eps):
    return v / np.sqrt((v * v).mean(-1, keepdims=True) + eps) * gamma


def rms_norm_backward(g, v, gamma, eps, gsum=None):
    """dx, dgamma."""
    d = np.sqrt((v * v).mean(-1, keepdims=True) + eps)
    h, a = v / d, g * gamma
    dx = (a - h * (a * h).mean(-1, keepdims=True)) / d
    return dx + (0.0 if gsum is None else gsum), (g * h).sum(0)
