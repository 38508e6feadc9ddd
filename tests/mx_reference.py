"""The block-scaled formats and products in 64 bits, from their definitions (numpy only)."""
from __future__ import annotations

import numpy as np

from paper_2512_13282_amd import inputs

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def widen(bits: np.ndarray) -> np.ndarray:
    with np.errstate(invalid="ignore"):     # signalling NaN patterns
        return inputs.f32_from_bf16_bits(bits).astype(np.float64)


def scale_values(e: np.ndarray) -> np.ndarray:
    return np.where(e == 255, np.nan, np.ldexp(1.0, e.astype(np.int64) - 127))


def pack(bits: np.ndarray, width: int) -> tuple[np.ndarray, np.ndarray]:
    """(codes, scales) of a matrix of bf16 bit patterns; width 4 or 8."""
    x = widen(bits)
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    scales = np.zeros((rows, nb), np.uint8)
    codes = np.zeros((rows, cols), np.int64)
    for r in range(rows):
        for b in range(nb):
            part = x[r, b * BLOCK:(b + 1) * BLOCK]
            if not np.all(np.isfinite(part)):
                scales[r, b] = 255
                continue
            big = np.max(np.abs(part))
            if big == 0:
                continue
            e = max(int(np.frexp(big)[1]) - 1 - (2 if width == 4 else 6), -127)
            scales[r, b] = e + 127
            v = np.ldexp(part, -e)
            if width == 8:
                q = np.clip(np.rint(v), -127, 127).astype(np.int64)
            else:
                # Distance to every code's value; a tie goes to the even code (mantissa bit 0).
                d = np.abs(np.abs(v)[:, None] - GRID[None, :])
                near = d == d.min(1, keepdims=True)
                even = near & (np.arange(8) % 2 == 0)
                q = np.where(even.any(1), even.argmax(1), near.argmax(1)) + 8 * np.signbit(v)
            codes[r, b * BLOCK:(b + 1) * BLOCK] = q
    if width == 8:
        return codes.astype(np.int8), scales
    codes = np.pad(codes, ((0, 0), (0, cols % 2)))
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8), scales


def values(codes: np.ndarray, scales: np.ndarray, cols: int) -> np.ndarray:
    """The matrix that packed codes stand for (uint8: 4 bits, int8: 8 bits)."""
    if codes.dtype == np.uint8:
        q = np.stack((codes & 15, codes >> 4), 2).reshape(codes.shape[0], -1)[:, :cols]
        v = np.where(q >= 8, -GRID[q & 7], GRID[q & 7])
    else:
        v = codes.astype(np.float64)
    return v * np.repeat(scale_values(scales), BLOCK, axis=1)[:, :cols]


def random_packed(rows: int, cols: int, width: int, seed: int) -> tuple[np.ndarray, np.ndarray]:
    """Codes of any bits (8-bit ones in [-127, 127]), scales around one."""
    rng = np.random.default_rng(seed)
    scales = rng.integers(120, 130, size=(rows, -(-cols // BLOCK))).astype(np.uint8)
    if width == 8:
        return rng.integers(-127, 128, size=(rows, cols)).astype(np.int8), scales
    return rng.integers(0, 256, size=(rows, (cols + 1) // 2)).astype(np.uint8), scales


def product(op: str, a: np.ndarray, b: np.ndarray) -> tuple[np.ndarray, np.ndarray]:
    """(C, sum of the terms' magnitudes) in 64 bits of fwd: a . b^T, dx: a . b, dw: a^T . b."""
    if op == "fwd":
        b = b.T
    if op == "dw":
        a = a.T
    return a @ b, np.abs(a) @ np.abs(b)


def bound(K: int, magnitude: np.ndarray, c: np.ndarray, bf16_out: bool) -> np.ndarray:
    """How far an fp32 sum of K exact products may be from the sum in 64 bits: each of at most
    K + 64 additions (64: more than the parts a sum is split into) loses at most one unit in the
    last place, 2^-23, of a partial sum, which is no larger than the terms' magnitudes together.  A
    rounding to bf16 adds half a unit of 2^-7, or half the spacing of bf16's subnormals."""
    t = (K + 64) * 2.0 ** -23 * magnitude
    return t + 2.0 ** -8 * (np.abs(c) + t) + 2.0 ** -134 if bf16_out else t + 2.0 ** -150
