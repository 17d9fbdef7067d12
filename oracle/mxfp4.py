"""Microscaled 4-bit floating point (E2M1 elements, one E8M0 scale for 32), in float64.

A block's scale is 2^(floor(log2 max|x|) - 2), at least 2^-127 (a block of zeros: 1; a
block with a non-finite value: NaN); an element is the representable multiple of it
nearest to x, ties to the even code, at most 6 in magnitude."""
from __future__ import annotations

import numpy as np

BLOCK = 32
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
MIDPOINTS = (MAGNITUDES[1:] + MAGNITUDES[:-1]) / 2


def round_code(a: np.ndarray) -> np.ndarray:
    """The code (0..7) nearest to each magnitude a >= 0; ties to the even code."""
    code = np.zeros(a.shape, dtype=np.int64)
    for i, mid in enumerate(MIDPOINTS):
        code += (a >= mid) if i % 2 else (a > mid)
    return code


def quantize(x: np.ndarray):
    """(codes 0..15 [rows, cols], scale bytes [rows, ceil(cols / 32)]) of blocks along the rows."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    blocks = (cols + BLOCK - 1) // BLOCK
    codes = np.zeros((rows, cols), dtype=np.uint8)
    scales = np.zeros((rows, blocks), dtype=np.uint8)
    for b in range(blocks):
        v = x[:, b * BLOCK:(b + 1) * BLOCK]
        top = np.max(np.abs(v), axis=1)
        bad = ~np.all(np.isfinite(v), axis=1)
        exp = np.zeros(rows, dtype=np.int64)
        fine = ~bad & (top > 0)
        exp[fine] = np.maximum(np.frexp(top[fine])[1] - 3, -127)
        scales[:, b] = np.where(bad, 255, exp + 127)
        with np.errstate(invalid="ignore"):
            c = round_code(np.abs(v) / np.exp2(exp)[:, None]) + 8 * np.signbit(v)
        codes[:, b * BLOCK:(b + 1) * BLOCK] = np.where(bad[:, None], 0, c)
    return codes, scales


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """What the codes stand for, float64."""
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    s = np.repeat(s, BLOCK, axis=1)[:, :codes.shape[1]]
    return np.where(codes >= 8, -1.0, 1.0) * MAGNITUDES[codes & 7] * s


def rounded(x: np.ndarray) -> np.ndarray:
    return values(*quantize(x))


def pack(codes: np.ndarray, scales: np.ndarray):
    """The stored form: bytes [rows, 64 groups], words of scale bytes [groups, rows, 4]."""
    rows, cols = codes.shape
    groups = (cols + 127) // 128
    full = np.zeros((rows, groups * 128), dtype=np.uint8)
    full[:, :cols] = codes
    s = np.full((rows, groups * 4), 127, dtype=np.uint8)
    s[:, :scales.shape[1]] = scales
    return full[:, 0::2] | full[:, 1::2] << 4, np.ascontiguousarray(s.reshape(rows, groups, 4).transpose(1, 0, 2))
