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


def buffer_bytes(code, scale):
    """The buffer of a matrix's [R, K] codes and [R, blocks] scale bytes: panels of 32 rows x 256
    columns, 4352 bytes each, zeros where there is nothing."""
    R, K = code.shape
    runs, slices = -(-R // 32), -(-K // 256)
    full = np.zeros((runs * 32, slices * 256), np.uint8)
    full[:R, :K] = code
    sc = np.zeros((runs * 32, slices * 8), np.uint8)
    sc[:R, :scale.shape[1]] = scale
    # [run, row, slice, half, ks, 16 pairs] -> [run, slice, ks, half, row, pair]
    pairs = (full[:, 0::2] | full[:, 1::2] << 4).reshape(runs, 32, slices, 2, 4, 16)
    values = pairs.transpose(0, 2, 4, 3, 1, 5).reshape(runs, slices, 4096)
    # [run, row, slice, half, ks] -> [run, slice, half, row, ks]
    scales = sc.reshape(runs, 32, slices, 2, 4).transpose(0, 2, 3, 1, 4).reshape(runs, slices, 256)
    return np.concatenate([values, scales], 2).reshape(-1)
