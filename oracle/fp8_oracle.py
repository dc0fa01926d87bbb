"""Copies in 8-bit floating point with a power of two for each block of 128, in float64 on the CPU.

codes(x, fmt, high): blocks of `high` rows (1, or 128 for a weight) by 128 columns; the scale byte of a block is 127 + the
least e >= -126 with max|x| <= F 2^e, or 255 where the block is not finite, and a code x 2^(127 - s) rounded to the
format, ties to even (0 where s = 255).
"""
import numpy as np

# largest number, bits of the mantissa, least exponent of a normal number
FORMATS = {"e4m3": (448.0, 3, -6), "e5m2": (57344.0, 2, -14)}


def pitch(cols):
    return (cols + 127) // 128 * 128


def scale_pitch(cols):
    return (cols + 2047) // 2048 * 16


def _round(t, fmt):
    """t (|t| <= F) to the nearest number of the format, ties to the even mantissa."""
    _, bits, least = FORMATS[fmt]
    _, e = np.frexp(t)
    step = np.exp2(np.maximum(e - 1, least) - bits)
    return np.where(t == 0, t, np.rint(t / step) * step)


def _byte(v, fmt):
    """Code bytes of numbers of the format."""
    _, bits, least = FORMATS[fmt]
    a = np.abs(v)
    _, e = np.frexp(a)
    e = np.where(a == 0, least, np.maximum(e - 1, least)).astype(int)
    m = (a / np.exp2(e - bits)).astype(np.int64)          # with the leading one, if there is one
    # a subnormal's exponent field is 0 and it has no leading one: e - least of it adds nothing
    code = ((e - least) << bits) + m
    return (code | np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)


def save(x, fmt="e4m3", high=1):
    """(code bytes [rows, pitch], scale bytes, values [rows, cols]) of x [rows, cols]."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    top = FORMATS[fmt][0]
    blocks_m, blocks_n = -(-rows // high), pitch(cols) // 128
    codes = np.zeros((rows, pitch(cols)), np.uint8)
    scales = np.ones((blocks_m, scale_pitch(cols)), np.uint8)
    values = np.zeros((rows, cols))
    for i in range(blocks_m):
        for j in range(blocks_n):
            at = (slice(i * high, min(rows, (i + 1) * high)), slice(128 * j, min(cols, 128 * j + 128)))
            b = x[at]
            if not np.all(np.isfinite(b)):
                scales[i, j] = 255
                values[at] = np.nan
                continue
            a = float(np.abs(b).max())
            e = -126
            if a > 0:
                e = int(np.frexp(a / top)[1]) - 1           # a / top = f 2^(e + 1), f in [1/2, 1)
                e = max(e if np.ldexp(top, e) >= a else e + 1, -126)
            q = _round(b * np.exp2(-float(e)), fmt)
            codes[at] = _byte(q, fmt)
            scales[i, j] = e + 127
            values[at] = q * np.exp2(float(e))
    return codes, scales, values


def load(codes, scales, fmt, cols, high=1):
    """The values that code and scale bytes stand for."""
    _, bits, least = FORMATS[fmt]
    c = codes.astype(np.int64)
    field, m = (c & 0x7F) >> bits, c & ((1 << bits) - 1)
    v = np.where(field == 0, m, m + (1 << bits)) * np.exp2(np.maximum(field - 1, 0) + least - bits)
    v = np.where(c & 0x80, -v, v)
    s = np.repeat(np.repeat(scales.astype(np.float64), high, 0)[:codes.shape[0]], 128, 1)[:, :codes.shape[1]]
    return np.where(s == 255, np.nan, v * np.exp2(np.where(s == 255, 127, s) - 127))[:, :cols]
