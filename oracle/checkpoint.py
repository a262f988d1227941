"""Oracle: rows kept in 8 bits (test infrastructure, CPU only).

Every 32 values of a row share a scale 2^e, e the smallest with max|x| <= 448 * 2^e (at least -126; 0 for a
group of zeros); a value is held as the e4m3 number nearest to x / 2^e, ties to the even one, of those that are below
2^128 with the scale.  The paper has no such
step; the format of the codes is the public 8-bit float with 4 exponent bits (bias 7), 3 mantissa bits and a
largest value of 448.
"""
import numpy as np

GROUP = 32


def e4m3_values():
    """The value of each of the 256 codes, from the format's fields."""
    out = np.empty(256)
    for code in range(256):
        sign = -1.0 if code & 0x80 else 1.0
        exponent, mantissa = (code >> 3) & 15, code & 7
        if exponent == 15 and mantissa == 7:
            out[code] = np.nan
        elif exponent == 0:
            out[code] = sign * mantissa * 2.0 ** -9
        else:
            out[code] = sign * (8 + mantissa) * 2.0 ** (exponent - 10)
    return out


def nearest_code(v):
    """Code of the e4m3 number nearest to each v (|v| <= 448; nan stays nan), by looking at all of them."""
    v = np.asarray(v, dtype=np.float64)
    values = e4m3_values()[:127]                         # 0 .. 448, ascending with the code
    a = np.abs(v)
    hi = np.clip(np.searchsorted(values, np.where(np.isnan(a), 0.0, a)), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = values[hi] - a, a - values[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    code = np.where(np.signbit(v), code + 128, code)
    return np.where(np.isnan(v), np.where(np.signbit(v), 255, 127), code).astype(np.uint8)


def store(x):
    """(codes [rows, d] uint8, biased exponents [rows, ceil(d / 32)] uint8); infinities and nan become nan."""
    x = np.asarray(x, dtype=np.float64)
    rows, d = x.shape
    groups = -(-d // GROUP)
    codes = np.empty((rows, d), np.uint8)
    scales = np.empty((rows, groups), np.uint8)
    for g in range(groups):
        part = x[:, g * GROUP:(g + 1) * GROUP]
        finite = np.isfinite(part)
        top = np.max(np.where(finite, np.abs(part), 0.0), axis=1)
        e = np.full(rows, -126)
        while np.any(top > 448.0 * 2.0 ** e):
            e = np.where(top > 448.0 * 2.0 ** e, e + 1, e)
        e = np.where(top == 0, 0, e)
        scales[:, g] = e + 127
        code = nearest_code(np.where(finite, part, np.nan) / (2.0 ** e)[:, None])
        over = finite & (np.abs(e4m3_values()[code]) * (2.0 ** e)[:, None] >= 2.0 ** 128)
        codes[:, g * GROUP:(g + 1) * GROUP] = code - over
    return codes, scales


def load(codes, scales):
    """The values a checkpoint stands for, fp64."""
    d = codes.shape[1]
    scale = 2.0 ** (scales.astype(np.float64) - 127)
    return e4m3_values()[codes] * np.repeat(scale, GROUP, axis=1)[:, :d]
