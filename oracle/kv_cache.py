"""The 8-bit cache format from its definition, with numpy: 4 exponent bits (bias 7), 3 mantissa bits, largest value 448, one
power of two per row."""
import numpy as np


def fp8_values():
    """The 127 non-negative finite values in order of their codes 0 .. 126."""
    code = np.arange(127)
    e, m = code >> 3, code & 7
    return np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))


def decode_fp8(codes):
    """uint8 codes -> float64 (code 127 of either sign: NaN)."""
    codes = np.asarray(codes, np.uint8)
    table = np.append(fp8_values(), np.nan)
    x = table[codes & 127]
    return np.where(codes >= 128, -x, x)


def quantise_rows(x):
    """x [..., D] -> (codes uint8 [..., D], exponents uint8 [...]): the smallest e >= -126 with max |x| <= 448 2^e over the finite
    elements; x / 2^e to the nearest value, of two as near the one with the even code; what is not finite becomes NaN."""
    x = np.asarray(x, np.float64)
    finite = np.isfinite(x)
    top = np.where(finite, np.abs(x), 0.0).max(axis=-1)
    e = np.full(top.shape, -126)
    while True:
        small = top > 448.0 * 2.0 ** e.astype(np.float64)
        if not small.any():
            break
        e = e + small
    y = np.where(finite, x, 0.0) / 2.0 ** e[..., None].astype(np.float64)
    grid = fp8_values()
    low = np.clip(np.searchsorted(grid, np.abs(y), side="right") - 1, 0, 125)
    below, above = np.abs(y) - grid[low], grid[low + 1] - np.abs(y)
    code = np.where((above < below) | ((above == below) & (low % 2 == 1)), low + 1, low)
    code = np.where(finite, code, 127)
    sign = np.signbit(np.where(np.isnan(x), 1.0, x))
    return (code + np.where(sign, 128, 0)).astype(np.uint8), (e + 127).astype(np.uint8)


def row_values(codes, exponents):
    return decode_fp8(codes) * 2.0 ** (np.asarray(exponents, np.float64)[..., None] - 127)


FP4_VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
FP4_GROUP = 32


def quantise_groups(x):
    """x [..., D] -> (bytes uint8 [..., D / 2], exponents uint8 [..., D / 32]) in 4 bits: per group of 32 elements the smallest e in -125 .. 125 with
    max |x| <= 6 2^e (none: 125); x / 2^e to the nearest value, of two as near the one with the even code, at most 6; the sign in the code's highest bit; two codes to a
    byte, the first in its low half.  A group with an element that is not finite: exponent 255, codes 0."""
    x = np.asarray(x, np.float64)
    y = x.reshape(*x.shape[:-1], -1, FP4_GROUP)
    fine = np.isfinite(y).all(axis=-1)
    y = np.where(fine[..., None], y, 0.0)
    top = np.abs(y).max(axis=-1)
    e = np.full(top.shape, -125)
    while True:
        small = (top > 6.0 * 2.0 ** e.astype(np.float64)) & (e < 125)
        if not small.any():
            break
        e = e + small
    y = y / 2.0 ** e[..., None].astype(np.float64)
    m = np.minimum(np.abs(y), 6.0)
    low = np.clip(np.searchsorted(FP4_VALUES, m, side="right") - 1, 0, 6)
    below, above = m - FP4_VALUES[low], FP4_VALUES[low + 1] - m
    code = np.where((above < below) | ((above == below) & (low % 2 == 1)), low + 1, low)
    code = np.where(fine[..., None], code + 8 * np.signbit(y), 0).astype(np.uint8).reshape(x.shape)
    return code[..., 0::2] | code[..., 1::2] << 4, np.where(fine, e + 127, 255).astype(np.uint8)


def group_values(codes, exponents):
    """float64 values [..., D] of bytes [..., D / 2] and exponents [..., D / 32]."""
    codes, e = np.asarray(codes, np.uint8), np.asarray(exponents, np.int64)
    both = np.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], -1)
    x = np.where(both >= 8, -1.0, 1.0) * FP4_VALUES[both & 7]
    scale = np.where(e == 255, np.nan, 2.0 ** (np.minimum(e, 254) - 127.0))
    return x * np.repeat(scale, FP4_GROUP, axis=-1)
