"""Microscaled formats in 64 bits: the definition, restated with numpy for the tests (TEST INFRASTRUCTURE ONLY).

Blocks of 32 consecutive values of a row share a scale 2^E.  Written from the formats' definition, element by
element where that is short, sharing nothing with the product package.
"""
from __future__ import annotations

import numpy as np

LEVELS4 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def bf16_values(bits: np.ndarray) -> np.ndarray:
    """uint16 bf16 bit patterns -> float64."""
    with np.errstate(invalid="ignore"):         # signalling NaNs
        return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def exponents(v: np.ndarray, below: int):
    """v float64 [rows, cols] -> int E [rows, blocks]; 128 where a value of the block is not finite."""
    rows, cols = v.shape
    blocks = -(-cols // BLOCK)
    E = np.empty((rows, blocks), dtype=np.int64)
    for b in range(blocks):
        part = np.abs(v[:, b * BLOCK:(b + 1) * BLOCK])
        with np.errstate(invalid="ignore"):
            top = part.max(axis=1)
        bad = ~np.isfinite(part).all(axis=1)
        mant, ex = np.frexp(np.where(bad, 1.0, top))     # top = mant * 2^ex, mant in [0.5, 1)
        e = np.maximum(np.where(top == 0, -127, ex - 1 - below), -127)
        E[:, b] = np.where(bad, 128, e)
    return E


def _spread(E, cols):
    s = np.where(E == 128, np.nan, np.ldexp(1.0, np.where(E == 128, 0, E)))
    return np.repeat(s, BLOCK, axis=1)[:, :cols]


def quantize4(v):
    """float64 [rows, cols] -> codes uint8 [rows, cols], E [rows, blocks]."""
    E = exponents(v, 2)
    with np.errstate(invalid="ignore"):
        a = np.abs(v) / _spread(E, v.shape[1])
    a = np.where(np.isnan(a), 0.0, a)
    dist = np.abs(np.minimum(a, 6.0)[..., None] - LEVELS4)
    near = dist.min(axis=-1, keepdims=True)
    hit = dist == near
    # of two equally near levels the one with the even code
    code = np.where(hit.sum(-1) == 2, np.where(hit.argmax(-1) % 2 == 0, hit.argmax(-1), hit.argmax(-1) + 1), hit.argmax(-1))
    code = code + 8 * np.signbit(v)
    return np.where(np.repeat(E == 128, BLOCK, axis=1)[:, :v.shape[1]], 0, code).astype(np.uint8), E


def values4(codes, E):
    sign = np.where(codes & 8, -1.0, 1.0)
    return sign * LEVELS4[codes & 7] * _spread(E, codes.shape[1])


def quantize8(v):
    E = exponents(v, 0)
    with np.errstate(invalid="ignore"):
        q = np.rint(v / _spread(E, v.shape[1]) * 64.0)
    q = np.clip(np.where(np.isnan(q), 0.0, q), -127, 127)
    return q.astype(np.int8), E


def values8(q, E):
    return q.astype(np.float64) / 64.0 * _spread(E, q.shape[1])


# ---- the library's layouts -----------------------------------------------------------------------------------
def pack4(codes, E):
    """Codes and scales as bytes: rows of whole blocks; tiles of 128 rows x 4 blocks of scales."""
    rows, cols = codes.shape
    blocks = E.shape[1]
    full = np.zeros((rows, blocks * BLOCK), dtype=np.uint8)
    full[:, :cols] = codes
    packed = full[:, 0::2] | full[:, 1::2] << 4
    tiles = -(-blocks // 4)
    scales = np.zeros((-(-rows // 128), tiles, 512), dtype=np.uint8)
    for i in range(rows):
        for b in range(blocks):
            scales[i // 128, b // 4, i % 32 * 16 + i % 128 // 32 * 4 + b % 4] = E[i, b] + 127
    return packed.reshape(-1), scales.reshape(-1)


def pack8(q, E):
    rows, cols = q.shape
    blocks = E.shape[1]
    full = np.zeros((rows, blocks * BLOCK), dtype=np.int8)
    full[:, :cols] = q
    e = np.zeros((rows, -(-blocks // 4) * 4), dtype=np.uint8)
    e[:, :blocks] = E + 127
    return full.view(np.uint8).reshape(-1), e.reshape(-1)
