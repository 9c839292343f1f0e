"""What a 4-bit cache holds in the place of 16-bit floats: codes and steps in exact arithmetic, values in 64 bits."""
from fractions import Fraction

import numpy as np

BITS = {"bfloat16": (8, -133, 128), "float16": (11, -24, 16)}  # of the significand, the least power of two, the first one too large


def round16(x, dtype, down=False):
    """Of finite numbers in 64 bits: the nearest on the type's grid, ties to even, or (x >= 0) the next one below."""
    bits, least, most = BITS[dtype]
    unit = np.ldexp(1.0, np.maximum(np.frexp(x)[1] - bits, least))
    y = np.asarray(x / unit)
    y = (np.floor(y) if down else np.rint(y)) * unit
    return np.where(np.abs(y) >= 2.0 ** most, np.copysign(np.inf, y), y)


def held(x, dtype):
    """Of the values x [.., D] in 64 bits (numbers of the type)."""
    x = np.asarray(x, np.float64)
    out = np.empty_like(x)
    for a in range(0, x.shape[-1], 32):
        y = x[..., a: a + 32]
        odd = ~np.isfinite(y).all(-1, keepdims=True)
        y = np.where(odd, 0.0, y)
        lo, hi = y.min(-1, keepdims=True), y.max(-1, keepdims=True)
        step = np.maximum(round16((hi - lo) / 15, dtype, down=True), 2.0 ** BITS[dtype][1])
        # y - lo as a sum of two floats, which is exact; a border between codes is a float, and the first one's place beside it is known
        t = y - lo
        rest = (y - (t - (t - y))) - (lo + (t - y))
        k = np.floor(t / step)
        border = (k + 0.5) * step
        on = (t == border) & (rest == 0)
        code = np.minimum(k + np.where(on, k % 2, (t > border) | ((t == border) & (rest > 0))), 15)
        out[..., a: a + 32] = np.where(odd, np.nan, round16(lo + code * step, dtype))
    return out


def held_exactly(x, dtype):
    """The same of one group, a list of numbers, in fractions."""
    x = [Fraction(v) for v in x]
    lo, hi = min(x), max(x)
    span = hi - lo
    if span == 0:
        return [float(lo)] * len(x)
    bits, least, _ = BITS[dtype]
    e = least
    while span / 15 >= Fraction(2) ** (e + bits):
        e += 1
    step = max((span / 15) // Fraction(2) ** e, 1) * Fraction(2) ** e
    out = []
    for v in x:
        code = min(round((v - lo) / step), 15)  # ties to even
        y = lo + code * step
        e = least
        while abs(y) >= Fraction(2) ** (e + bits):
            e += 1
        out.append(float(round(y / Fraction(2) ** e) * Fraction(2) ** e))
    return out
