"""Reference of the 8-bit cache's format and of rotary positions, in 64 bits and numpy.  TEST INFRASTRUCTURE ONLY: it
imports nothing from the product package.

Written from the definitions: a code is sign, 4 bits of exponent (bias 7), 3 of significand; exponent 0 is
subnormal; all ones is NaN; there are no infinities.  A row's scale is the least power of two, at least 2^-117, that
brings its largest finite magnitude to 448 or below, or 2^119; larger values are held as 448 times that."""
from __future__ import annotations

import numpy as np

LEAST_EXPONENT, MOST_EXPONENT, BIAS, LARGEST = -117, 119, 127, 448.0


def code_values() -> np.ndarray:
    """The value of each of the 256 codes (NaN for 0x7f and 0xff)."""
    code = np.arange(256)
    exponent, significand = (code >> 3) & 15, code & 7
    value = np.where(exponent == 0, significand / 8.0 * 2.0 ** -6, (1 + significand / 8.0) * 2.0 ** (exponent - 7.0))
    value = np.where((code & 0x7F) == 0x7F, np.nan, value)
    return np.where(code >> 7, -value, value)


def row_exponents(x: np.ndarray) -> np.ndarray:
    """e of every row along the last axis."""
    most = np.where(np.isfinite(x), np.abs(x), 0.0).max(axis=-1)
    e = np.full(most.shape, LEAST_EXPONENT, np.int64)
    while True:                                              # the least one that holds, by trying
        short = (most > LARGEST * 2.0 ** e) & (e < MOST_EXPONENT)
        if not short.any():
            return e
        e[short] += 1


def quantise(x: np.ndarray):
    """Rows along the last axis -> (codes uint8, scale bytes uint8).  Nearest code, by distance to all 127 magnitudes' neighbours;
    ties to the even code."""
    x = np.asarray(x, np.float64)
    e = row_exponents(x)
    y = x / (2.0 ** e)[..., None]
    values = code_values()[:0x7F]                            # 0 .. 448, rising
    size = np.minimum(np.abs(np.where(np.isfinite(y), y, 0.0)), LARGEST)
    hi = np.clip(np.searchsorted(values, size), 1, 0x7E)
    lo = hi - 1
    below, above = size - values[lo], values[hi] - size
    code = np.where((above < below) | ((above == below) & (hi % 2 == 0)), hi, lo).astype(np.uint8)
    code = np.where(np.signbit(y), code | 0x80, code)
    code = np.where(np.isfinite(y), code, 0x7F).astype(np.uint8)
    return code, (e + BIAS).astype(np.uint8)


def values_of(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    return code_values()[codes] * (2.0 ** (scales.astype(np.float64) - BIAS))[..., None]


def rotate(x: np.ndarray, positions: np.ndarray, inv_freq: np.ndarray, rotary_dim: int, layout: str, factor: float = 1.0,
           inverse: bool = False) -> np.ndarray:
    """x [T][heads][d]; positions [T][rotary_dim / 2] (each frequency's own) -> rotated, in 64 bits."""
    x = np.array(x, np.float64)
    angle = positions.astype(np.float64) * inv_freq * (-1.0 if inverse else 1.0)
    turn = (factor * np.exp(1j * angle))[:, None, :]
    pick = (slice(0, rotary_dim // 2), slice(rotary_dim // 2, rotary_dim)) if layout == "half" else (slice(0, rotary_dim, 2), slice(1, rotary_dim, 2))
    z = (x[..., pick[0]] + 1j * x[..., pick[1]]) * turn
    x[..., pick[0]], x[..., pick[1]] = z.real, z.imag
    return x
