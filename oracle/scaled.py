"""8-bit block-scaled matrices, in fp64 numpy: codes, values and products.

A code is the nearest value of its type to x * (1 / scale), ties to even, with
scale = max(max |x| / M, 2^-100) over blocks of 128 columns and 1 or 128 rows.
The scale, its reciprocal and the product are fp32 by definition (numpy's fp32
operations round to nearest, as IEEE asks); the rounding to a code is done here
in fp64 from the definition of the type.
"""

from __future__ import annotations

import numpy as np

BLOCK = 128
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
BITS = {"e4m3": (3, -6), "e5m2": (2, -14)}   # mantissa bits, exponent of the least normal value
LEAST = np.float32(2.0 ** -100)


def step_of(y: np.ndarray, code: str) -> np.ndarray:
    """Distance between neighbouring codes around |y|."""
    bits, least = BITS[code]
    _, e = np.frexp(np.abs(y))          # |y| in [2^(e-1), 2^e)
    return np.exp2(np.maximum(e - 1, least) - bits).astype(np.float64)


def round_to_code(y: np.ndarray, code: str) -> np.ndarray:
    y = np.asarray(y, dtype=np.float64)
    s = step_of(y, code)
    return np.rint(y / s) * s           # (numpy's rint: ties to even)


def encode(values: np.ndarray, code: str) -> np.ndarray:
    """uint8 bits of values that are codes."""
    bits, least = BITS[code]
    bias = 1 - least
    a = np.abs(values)
    _, e = np.frexp(a)
    normal = a >= 2.0 ** least
    m = np.where(normal, a / np.exp2(e - 1.0) - 1.0, a / 2.0 ** least) * 2 ** bits
    field = np.where(normal, e - 1 + bias, 0)
    return (np.signbit(values).astype(np.uint8) << 7) | (field.astype(np.int64) << bits).astype(np.uint8) | m.astype(np.uint8)


def decode(bits: np.ndarray, code: str) -> np.ndarray:
    mb, least = BITS[code]
    b = bits.astype(np.int64)
    e, m = (b >> mb) & ((1 << (7 - mb)) - 1), b & ((1 << mb) - 1)
    v = np.where(e > 0, (1 + m / 2.0 ** mb) * np.exp2(e - 1.0 + least), m / 2.0 ** mb * 2.0 ** least)
    return np.where(b >> 7, -v, v)


def _blocks(a: np.ndarray, block_rows: int) -> np.ndarray:
    """Maximum of |a| per block, [column blocks][row blocks]."""
    rows, cols = a.shape
    rb, cb = -(-rows // block_rows), -(-cols // BLOCK)
    p = np.zeros((rb * block_rows, cb * BLOCK), dtype=a.dtype)
    p[:rows, :cols] = np.abs(a)
    return np.ascontiguousarray(p.reshape(rb, block_rows, cb, BLOCK).max(axis=(1, 3)).T)


def expand(scale: np.ndarray, rows: int, cols: int, block_rows: int) -> np.ndarray:
    return np.repeat(np.repeat(scale.T, block_rows, axis=0), BLOCK, axis=1)[:rows, :cols]


def quantize(x: np.ndarray, block_rows: int, code: str):
    """(values of the codes [rows][cols], fp32 scales [column blocks][row blocks]) of an fp32 matrix."""
    x = np.asarray(x, dtype=np.float32)
    scale = np.maximum(_blocks(x, block_rows) / np.float32(LARGEST[code]), LEAST)
    inverse = np.float32(1.0) / scale
    return round_to_code(x * expand(inverse, *x.shape, block_rows), code), scale


def values(codes: np.ndarray, scale: np.ndarray, block_rows: int) -> np.ndarray:
    return codes * expand(scale.astype(np.float64), *codes.shape, block_rows)


def matmul(a: np.ndarray, b: np.ndarray):
    """A B^T of two matrices of values, and the sum of the terms' magnitudes."""
    return a @ b.T, np.abs(a) @ np.abs(b).T
