"""What the 8-bit block store holds, from its definition, in numpy and 64 bits (no code of the library)."""
import numpy as np

# The values of the 256 codes: sign, 4 bits of exponent (bias 7), 3 of mantissa; 0x7F and 0xFF are NaN.
CODES = np.array([(-1.0 if c & 128 else 1.0) * ((c & 7) * 2.0 ** -9 if (c >> 3 & 15) == 0 else (8 + (c & 7)) * 2.0 ** ((c >> 3 & 15) - 10))
                  if c & 127 != 127 else np.nan for c in range(256)])


def scale_exponents(x):
    """e of every row of x [..., D]: the least whole e >= -111 with max |finite x| <= 448 * 2^e."""
    top = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1).astype(np.float64)
    e = np.full(top.shape, -111)
    while True:
        low = top > 448.0 * 2.0 ** e.astype(np.float64)
        if not low.any():
            return e
        e = e + low


def round_to_codes(y):
    """y to the nearest value of a code, ties to the even code; NaN where y is not finite."""
    grid = CODES[:127]                                # 0 .. 448, ascending: code number = place
    a = np.abs(y)
    hi = np.clip(np.searchsorted(grid, np.where(np.isfinite(a), a, 0.0)), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - a, a - grid[lo]
    take_hi = (up < down) | ((up == down) & (hi % 2 == 0))
    v = np.where(take_hi, grid[hi], grid[lo])
    return np.where(np.isfinite(y), np.copysign(v, y), np.nan)


def held(x):
    """What the store gives back for rows x [..., D]."""
    x = np.asarray(x, dtype=np.float64)
    s = 2.0 ** scale_exponents(x).astype(np.float64)[..., None]
    v = round_to_codes(x / s) * s
    most = 240.0 * 2.0 ** 120                         # the next larger code would stand for 2^128
    return np.where(np.abs(v) > most, np.where(s == 2.0 ** 120, np.copysign(most, v), v), v)
