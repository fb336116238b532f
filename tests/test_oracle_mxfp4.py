"""Pins of the MXFP4 oracle: the format's numbers, its rounding by brute force, its scale's
closed forms, and the buffer's places counted one by one."""

import math

import numpy as np
import pytest

from oracle import mxfp4 as mx


def test_sizes_from_the_bit_fields():
    """E2M1: exponent bias 1, one mantissa bit, subnormals at exponent 0."""
    for code, size in enumerate(mx.SIZES):
        exp, man = code >> 1, code & 1
        assert size == (math.ldexp(man, -1) if exp == 0 else math.ldexp(1 + man / 2, exp - 1))


def test_rounding_against_every_neighbour():
    """Nearest of all eight; at each midpoint the even code; past 6 the largest."""
    for lo, hi in zip(range(7), range(1, 8)):
        mid = (mx.SIZES[lo] + mx.SIZES[hi]) / 2
        even = lo if lo % 2 == 0 else hi
        got = mx.codes([mid - 1e-9, mid, mid + 1e-9, mx.SIZES[lo], mx.SIZES[hi]])
        assert got.tolist() == [lo, even, hi, lo, hi]
    assert mx.codes([6.0, 7.0, 7.999, 0.0]).tolist() == [7, 7, 7, 0]


@pytest.mark.parametrize("top,e", [(1.0, -2), (1.999, -2), (2.0, -1), (6.0, 0), (7.99, 0), (8.0, 1),
                                   (0.75, -3), (0.0, -127), (2.0 ** -125, -127), (2.0 ** -124, -126),
                                   (1e-44, -127), (3.4e38, 125)])
def test_scale(top, e):
    block = np.zeros(32)
    block[5] = -top
    assert mx.exponent(block) == e


def test_values_are_near_and_idempotent():
    x = np.random.default_rng(0).normal(size=(5, 100)) * 10.0 ** np.arange(-2, 3)[:, None]
    v, code, scale = mx.quantize(x)
    for r in range(5):
        for b in range(4):
            e = int(scale[r, b]) - 127
            at = slice(32 * b, min(32 * b + 32, 100))
            # half the widest gap, and 2 where sizes of up to 8 saturate at 6
            assert np.all(np.abs(v[r, at] - x[r, at]) <= 2.0 * 2.0 ** e)
            small = np.abs(x[r, at]) <= 6 * 2.0 ** e
            assert np.all(np.abs(v[r, at] - x[r, at])[small] <= 2.0 ** e)
    again = mx.quantize(v)
    assert np.array_equal(again[0], v)
    bad = x.copy()
    bad[2, 40], bad[3, 99] = np.inf, np.nan
    w, _, s = mx.quantize(bad)
    assert np.isnan(w[2, 32:64]).all() and np.isnan(w[3, 96:]).all() and np.isfinite(w[2, :32]).all()
    assert s[2, 1] == 255 and s[3, 3] == 255


def test_buffer_place_by_place():
    R, K = 35, 300
    rng = np.random.default_rng(1)
    code = rng.integers(1, 16, (R, K)).astype(np.uint8)
    scale = rng.integers(1, 255, (R, 10)).astype(np.uint8)
    q = mx.buffer_bytes(code, scale)
    assert q.size == 2 * 2 * 4352
    left = q.copy()
    for r in range(R):
        for k in range(K):
            b, j = k % 256 // 32, k % 32
            at = (r // 32 * 2 + k // 256) * 4352 + b % 4 * 1024 + (b // 4 * 32 + r % 32) * 16 + j // 2
            assert q[at] >> (4 * (j % 2)) & 15 == code[r, k]
            left[at] &= 0xF0 if j % 2 == 0 else 0x0F
        for b in range(10):
            at = (r // 32 * 2 + b // 8) * 4352 + 4096 + (b % 8 // 4 * 32 + r % 32) * 4 + b % 4
            assert q[at] == scale[r, b]
            left[at] = 0
    assert not left.any()
