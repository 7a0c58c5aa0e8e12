"""Norms of queries and keys, head by head, with their rotation by position, and the gradients, in fp64 from the formulas.

Limits on the errors of a computation in fp32, in units of F = 2^-24, half a step of fp32 (each operation rounds by at most that, relative to its result):
  r = 1 / sqrt(mean x^2 + eps): up to 20 roundings in a row in a sum of squares (16 in a lane, 3 across lanes, 1 with eps), which have one sign: 20 F, of
      which the root leaves half; root and reciprocal 4: 14 F.  n = x r w: 3 more, 17 F.
  sine and cosine: the fraction of a turn is rounded to fp32, an angle of up to pi by pi F, and the functions by 4 F: 8 F absolute.
  a pair (a, b): 17 + 8 + 3 of products and their sum: 28 F (|a| + |b|).  Taken as 32.
  backward: a rotated pair 11 F (|a| + |b|), times w, the unit row x r (16) and a sum of up to 20 terms in a row: 48 F of the sum of
      magnitudes; dx = r (dn w - x r mean): 14 + 3 more.  Taken as 72 for dx.  A weight's gradient adds `chain` terms in a row: (32 + chain) F of
      the sum of magnitudes.
The result's rounding comes on top: half a step of its type, `half` relative."""
import numpy as np

F = 2.0 ** -24


def _pairs(rotary, interleaved):
    i = np.arange(rotary // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)


def _turn(x, angle, rotary, interleaved):
    """x [n, heads, D], angle [n, R / 2]; also the sums of magnitudes |a| + |b| that each result is made of."""
    y, size = x.copy(), np.abs(x)
    a, b = _pairs(rotary, interleaved)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y, size


TURN = 159154943091895335768883763372514362034459645740456448747667344058896797634226535        # 10^81 / (2 pi)


def _angle(positions, inv_freq):
    """In whole numbers: the turns, of which a position has 2^200 f / (2 pi) parts of 2^-200, lose their whole ones, and what is left is a number of 64 bits."""
    ratios = [float(f).as_integer_ratio() for f in np.asarray(inv_freq)]
    per = np.array([(a * TURN << 200) // (b * 10 ** 81) for a, b in ratios], dtype=object)
    half = np.array([1 << 199], dtype=object)
    parts = (np.asarray(positions).astype(np.int64).astype(object)[:, None] * per + half) % (2 * half) - half
    return 2 * np.pi * ((parts // 2 ** 137).astype(np.float64) * 2.0 ** -63)


def norm_rotate(x, w=None, positions=None, inv_freq=None, eps=1e-6, interleaved=False, half=0.0):
    """x [n, heads, D] -> (results, limits on their errors)."""
    x = np.asarray(x, np.float64)
    n = x
    if w is not None:
        n = x / np.sqrt(np.square(x).mean(-1, keepdims=True) + eps) * np.asarray(w, np.float64)
    size = np.abs(n)
    if inv_freq is not None and len(inv_freq):
        n, size = _turn(n, _angle(positions, inv_freq), 2 * len(inv_freq), interleaved)
    return n, 32 * F * size + half * (1 + 2 ** -8) * np.abs(n)


def norm_rotate_backward(dout, x, w=None, positions=None, inv_freq=None, eps=1e-6, interleaved=False, half=0.0, chain=64):
    """dict(dx, e_dx, and with a weight dw, e_dw)."""
    x, dn = np.asarray(x, np.float64), np.asarray(dout, np.float64)
    size = np.abs(dn)
    if inv_freq is not None and len(inv_freq):
        dn, size = _turn(dn, -_angle(positions, inv_freq), 2 * len(inv_freq), interleaved)
    if w is None:
        return dict(dx=dn, e_dx=32 * F * size + half * (1 + 2 ** -8) * np.abs(dn))
    w = np.asarray(w, np.float64)
    r = 1 / np.sqrt(np.square(x).mean(-1, keepdims=True) + eps)
    unit = x * r
    dx = r * (dn * w - unit * (dn * w * unit).mean(-1, keepdims=True))
    terms = r * (size * np.abs(w) + np.abs(unit) * (size * np.abs(w * unit)).mean(-1, keepdims=True))
    return dict(dx=dx, e_dx=72 * F * terms + half * (1 + 2 ** -8) * np.abs(dx), dw=(dn * unit).sum((0, 1)),
                e_dw=(32 + chain) * F * (size * np.abs(unit)).sum((0, 1)))
