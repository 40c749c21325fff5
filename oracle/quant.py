"""Rows of an 8-bit cache, in float64 (test infrastructure).

A row is 128 OCP E4M3 codes (4 exponent bits of bias 7, 3 fraction bits, no
infinities, largest finite value 448) and one power of two 2^s.  With amax = f *
2^e, 1 <= f < 2, the largest |x_c| of the row, s = e - 8 where f <= 1.75 and e - 7
above, at least -126; the codes are x_c / 2^s rounded to nearest, ties to the even
code, within +-448, or within +-240 where s = 120 (256 * 2^120 is past the largest
bf16 number).  An infinity counts as the largest bf16 number; a NaN stays a NaN and
has no part in amax.
"""

import numpy as np

BF16_MAX = float(2.0 ** 127 * (2 - 2.0 ** -7))


def e4m3_values():
    """The values of codes 0 .. 126 (127 is NaN), ascending."""
    out = []
    for code in range(127):
        e, f = code >> 3, code & 7
        out.append(f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10))
    return np.array(out)


_GRID = e4m3_values()


def round_e4m3(y, limit=448.0):
    """|y| to the nearest grid value, ties to the even code, the sign kept."""
    a = np.minimum(np.abs(y), limit)
    hi = np.searchsorted(_GRID, a)                 # first code >= a
    hi = np.minimum(hi, len(_GRID) - 1)
    lo = np.maximum(hi - 1, 0)
    below, above = a - _GRID[lo], _GRID[hi] - a
    up = (above < below) | ((above == below) & (hi % 2 == 0))
    return np.copysign(np.where(up, _GRID[hi], _GRID[lo]), y)


def row_exponent(amax):
    f, e = np.frexp(amax)                          # amax = 2f * 2^(e-1)
    s = np.where(2 * f <= 1.75, e - 9, e - 8)
    return np.maximum(np.where(amax == 0, -126, s), -126)


def held_rows(x):
    """The values that rows [..., d] stand for once held, float64."""
    x = np.asarray(x, dtype=np.float64)
    nan = np.isnan(x)
    y = np.clip(np.where(nan, 0.0, x), -BF16_MAX, BF16_MAX)
    s = row_exponent(np.abs(y).max(-1, keepdims=True))
    limit = np.where(s == 120, 240.0, 448.0)
    out = round_e4m3(y / 2.0 ** s, limit) * 2.0 ** s
    return np.where(nan, np.nan, out)
