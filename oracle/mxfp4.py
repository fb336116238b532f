"""MXFP4 in float64, from the format's definition: blocks of 32 values along a row, a scale
2^e per block, values from the fifteen numbers of E2M1."""

from __future__ import annotations

import math

import numpy as np

#: the sizes of E2M1 by code (two exponent bits, one mantissa bit)
SIZES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def exponent(block):
    """e of a block of finite values: floor(log2) of the largest size less 2 (the exponent of
    the format's largest number), not below -127; None for a block with an infinity or a NaN."""
    top = float(np.max(np.abs(block), initial=0.0))
    if not math.isfinite(top):
        return None
    return -127 if top == 0.0 else max(math.frexp(top)[1] - 1 - 2, -127)


def codes(size):
    """The code of the nearest size for each entry of `size` (>= 0), of two as near the even one,
    beyond the largest the largest."""
    gap = np.abs(np.asarray(size, np.float64)[..., None] - SIZES)
    least = gap.min(-1, keepdims=True)
    tied = gap == least  # at most two, neighbours
    first = tied.argmax(-1)
    both = tied.sum(-1) == 2
    return np.where(both & (first % 2 == 1), first + 1, first)


def quantize(x):
    """(values, code bytes, exponents) of a matrix: float64 [R, K] values that its four-bit form
    stands for, uint8 [R, K] codes with the sign in bit 3, and [R, ceil(K / 32)] E8M0 bytes."""
    x = np.asarray(x, np.float64)
    R, K = x.shape
    nb = -(-K // BLOCK)
    values, code = np.empty((R, K)), np.empty((R, K), np.uint8)
    scale = np.empty((R, nb), np.uint8)
    for b in range(nb):
        part = x[:, b * BLOCK:(b + 1) * BLOCK]
        at = slice(b * BLOCK, b * BLOCK + part.shape[1])
        for r in range(R):
            e = exponent(part[r])
            if e is None:
                values[r, at], code[r, at], scale[r, b] = np.nan, 0, 255
                continue
            c = codes(np.abs(part[r]) * 2.0 ** -e)
            neg = np.signbit(part[r])
            code[r, at] = c | neg.astype(np.uint8) << 3
            values[r, at] = np.where(neg, -1.0, 1.0) * SIZES[c] * 2.0 ** e
            scale[r, b] = e + 127
    return values, code, scale


def packed_bytes(code):
    """The packed buffer of a matrix's codes: two a byte, the even column low, rows padded with
    zeros to 256 columns."""
    R, K = code.shape
    full = np.zeros((R, -(-K // 256) * 256), np.uint8)
    full[:, :K] = code
    return full[:, 0::2] | full[:, 1::2] << 4


def scale_bytes(scale):
    """The scale buffer of a matrix's [R, blocks] scale bytes: per slice of 8 blocks and run of 32
    rows 256 bytes, block b of row r at (b % 8 // 4) * 128 + r % 32 * 4 + b % 4; zeros elsewhere."""
    R, nb = scale.shape
    slices, runs = -(-nb // 8), -(-R // 32)
    out = np.zeros((slices, runs, 256), np.uint8)
    r, b = np.meshgrid(np.arange(R), np.arange(nb), indexing="ij")
    out[b // 8, r // 32, b % 8 // 4 * 128 + r % 32 * 4 + b % 4] = scale
    return out.reshape(-1)
