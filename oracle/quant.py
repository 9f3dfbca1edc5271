"""A cache held in 8 bits: quantising blocks of rows, and what the codes stand for.

The scale of a block of rows and head is 2^e with the least e >= -100 for which the
largest magnitude is at most most * 2^e (most: 448 for e4m3, 127 for int8); a code is the
representable value nearest to x / 2^e, of two equally near the even one.  A block with a
value that is not finite has the scale NaN and codes 0.  So that code * 2^e stays within
fp32, e4m3 codes end at 240 where e is 120 and int8 codes at 63 where e is 122.
"""
import numpy as np

MOST = {"e4m3": 448.0, "int8": 127.0}


def e4m3_values():
    """The values of the e4m3 codes 0 .. 126, which rise with the code."""
    out = []
    for code in range(127):
        exponent, mantissa = code >> 3, code & 7
        out.append(mantissa / 8 * 2.0 ** -6 if exponent == 0 else
                   (1 + mantissa / 8) * 2.0 ** (exponent - 7))
    return np.array(out)


def scale_exponent(top, fmt):
    """The least e >= -100 with top <= most * 2^e."""
    e = -100
    while top > MOST[fmt] * 2.0 ** e:
        e += 1
    return e


def nearest(x, fmt):
    """The nearest values of a format; of two equally near, the one with the even code."""
    if fmt == "int8":
        return np.rint(x)
    table = e4m3_values()
    a = np.abs(x)
    up = np.clip(np.searchsorted(table, a), 1, 126)
    lo, hi = table[up - 1], table[up]
    down = (a - lo < hi - a) | ((a - lo == hi - a) & ((up - 1) % 2 == 0))
    return np.copysign(np.where(down, lo, hi), x)


def quantize(X, block, fmt):
    """X [n, rows, H, d] -> codes (as values) [n, H, rows, d], scales [n, H, ceil(rows /
    block)]."""
    n, rows, H, d = X.shape
    codes = np.zeros((n, H, rows, d))
    scales = np.zeros((n, H, -(-rows // block)))
    for i, h, b in np.ndindex(*scales.shape):
        x = X[i, b * block:(b + 1) * block, h].astype(np.float64)
        if not np.isfinite(x).all():
            scales[i, h, b] = np.nan
            continue
        e = scale_exponent(np.abs(x).max(), fmt)
        scales[i, h, b] = 2.0 ** e
        c = nearest(x / 2.0 ** e, fmt)
        if (fmt, e) == ("e4m3", 120):
            c = np.clip(c, -240, 240)
        if (fmt, e) == ("int8", 122):
            c = np.clip(c, -63, 63)
        codes[i, h, b * block:(b + 1) * block] = c
    return codes, scales


def values(codes, scales, block):
    """What codes [n, H, rows, d] stand for: [n, rows, H, d]."""
    rows = codes.shape[2]
    s = np.repeat(scales, block, axis=2)[:, :, :rows, None]
    return np.swapaxes(codes * s, 1, 2)
