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
