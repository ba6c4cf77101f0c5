"""Oracle for the microscaled 4-bit format and the sorting of slots by expert.

TEST INFRASTRUCTURE ONLY -- never called by the product.

E2M1: 1 sign bit, 2 exponent bits with bias 1, 1 mantissa bit, no infinities or NaN.  E8M0:
2^(code - 127), 255 NaN.  Everything is computed in 64 bits from the definitions: the scale
of a block of 32 is 2^(floor(log2 max|x|) - 2), at least 2^-127 (NaN if the block holds an
infinity or NaN), an element the nearest E2M1 value of x over the scale, ties to the even
code, saturating at 6.
"""
from __future__ import annotations

import numpy as np

BLOCK = 32


def e2m1_value(code: int) -> float:
    """Value of one E2M1 code, from the format's definition."""
    sign = -1.0 if code & 8 else 1.0
    e, m = (code >> 1) & 3, code & 1
    return sign * (m * 0.5 if e == 0 else (1 + m * 0.5) * 2.0 ** (e - 1))


GRID = np.array([e2m1_value(c) for c in range(16)])


def e8m0_value(codes: np.ndarray) -> np.ndarray:
    codes = np.asarray(codes, dtype=np.int64)
    return np.where(codes == 255, np.nan, np.ldexp(1.0, np.where(codes == 255, 0, codes - 127)))


def quantise(x: np.ndarray):
    """(codes, scales) of a float64 matrix, blocks along the rows: uint8 (rows, 32*blocks), one
    code to an entry, and uint8 (rows, blocks)."""
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    b = np.zeros((rows, blocks * BLOCK))
    b[:, :cols] = x
    b = b.reshape(rows, blocks, BLOCK)
    bad = ~np.isfinite(b).all(axis=2)
    b = np.where(bad[..., None], 0.0, b)
    top = np.abs(b).max(axis=2)
    _, exponent = np.frexp(top)                      # top = m * 2^exponent, m in [0.5, 1)
    s = np.where(top == 0, 0, np.clip(exponent - 1 - 2 + 127, 0, 254))
    m = np.abs(b) / e8m0_value(s)[..., None]
    code = np.zeros(m.shape, dtype=np.int64)
    for i in range(7):
        middle = (GRID[i] + GRID[i + 1]) / 2
        code += (m > middle) | ((m == middle) & (i % 2 == 1))
    code += 8 * np.signbit(b)
    return code.reshape(rows, -1).astype(np.uint8), np.where(bad, 255, s).astype(np.uint8)


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """float64 values of unpacked codes and their scales."""
    return GRID[codes] * np.repeat(e8m0_value(scales), BLOCK, axis=-1)


def pack(codes: np.ndarray) -> np.ndarray:
    """Two codes to a byte, the even column in the low bits."""
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(packed: np.ndarray) -> np.ndarray:
    out = np.empty(packed.shape[:-1] + (packed.shape[-1] * 2,), dtype=np.uint8)
    out[..., 0::2] = packed & 15
    out[..., 1::2] = packed >> 4
    return out


def sort_slots(ids: np.ndarray, experts: int, align: int, rows: int):
    """(offsets, order, pos) of a stable sort of the slots by expert."""
    order, offsets = [], [0]
    pos = np.full(ids.size, -1, dtype=np.int32)
    flat = ids.reshape(-1)
    for e in range(experts):
        slots = [s for s in range(flat.size) if flat[s] == e]
        for i, s in enumerate(slots):
            pos[s] = offsets[-1] + i
        order += slots + [-1] * (-len(slots) % align)
        offsets.append(len(order))
    order += [-1] * (rows - len(order))
    return np.array(offsets, dtype=np.int32), np.array(order, dtype=np.int32), pos
