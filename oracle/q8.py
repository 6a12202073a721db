"""Matrices in 8 bits, in fp64: codes are floats of 4 exponent bits (bias 7) and 3
fraction bits, in units of the power of two (2^-126 at least) that puts the largest
finite magnitude of 128 elements of a row, or of a tile of 128 x 128, into [128, 256).
"""

import numpy as np

BLOCK = 128


def value(code):
    """What 8-bit codes stand for; 0x7F and 0xFF are NaN."""
    code = np.asarray(code, np.uint8).astype(np.int64)
    e, m = (code >> 3) & 15, code & 7
    v = np.where(e > 0, (8.0 + m) * 2.0 ** (e - 10.0), m * 2.0 ** -9)
    v = np.where((code & 127) == 127, np.nan, v)
    return np.where(code & 128, -v, v)


def nearest(x):
    """The nearest of those values to x, |x| < 256 or not finite (halves to even)."""
    x = np.asarray(x, np.float64)
    mag = np.where(np.isfinite(x), np.abs(x), 0.0)
    unit = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(mag, 2.0 ** -20))), -6) - 3)
    return np.where(np.isfinite(x), np.sign(x) * np.rint(mag / unit) * unit, np.nan)


def exponents(x, tiles=False):
    """The scales' exponent bytes, [rows or tiles][blocks of 128 columns]."""
    x = np.asarray(x, np.float64)
    R, C = x.shape
    rows = BLOCK if tiles else 1
    mag = np.zeros((-(-R // rows) * rows, -(-C // BLOCK) * BLOCK))
    mag[:R, :C] = np.where(np.isfinite(x), np.abs(x), 0.0)
    top = mag.reshape(mag.shape[0] // rows, rows, mag.shape[1] // BLOCK, BLOCK).max((1, 3))
    e = np.floor(np.log2(np.maximum(top, 2.0 ** -200))).astype(np.int64) + 127 - 7
    return np.maximum(e, 1).astype(np.uint8)


def spread(e, shape, tiles=False):
    """The scale of every element of a matrix of this shape."""
    s = np.repeat(2.0 ** (np.asarray(e, np.float64) - 127), BLOCK, 1)[:, :shape[1]]
    return np.repeat(s, BLOCK, 0)[:shape[0]] if tiles else s


def quantise(x, tiles=False):
    """(values of the codes, exponent bytes)."""
    e = exponents(x, tiles)
    return nearest(np.asarray(x, np.float64) / spread(e, np.shape(x), tiles)), e
