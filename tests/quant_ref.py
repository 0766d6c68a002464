"""The 8-bit prefix cache in 64 bits, written from its definition: numpy only, shares nothing with the kernels."""
import math

import numpy as np

BLOCK = 64


def code_values():
    """Value of each e4m3 code: sign, 4 bits of exponent with bias 7, 3 bits of mantissa; 0x7f and 0xff are NaN."""
    v = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        a = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[c] = math.copysign(math.nan if c & 127 == 127 else a, -1.0 if c >> 7 else 1.0)
    return v


VALUES = code_values()


def scale_of(x):
    """The smallest 2^e with max |x| <= 448 * 2^e among finite x, -117 <= e <= 119."""
    a = np.abs(x[np.isfinite(x)])
    top = a.max() if a.size else 0.0
    e = -117
    while top > 448.0 * 2.0 ** e and e < 119:
        e += 1
    return 2.0 ** e


def encode(x, s):
    """Codes of x / s: the nearest value, the even code of two; magnitudes above 448 and infinities the largest code."""
    y = np.asarray(x, np.float64) / s
    a = np.minimum(np.abs(y), 448.0)
    with np.errstate(divide="ignore", invalid="ignore"):
        step = np.exp2(np.maximum(np.floor(np.log2(a)), -6) - 3)
    r = np.rint(np.where(a == 0, 0, a / step)) * step
    code = np.searchsorted(VALUES[:127], np.where(np.isnan(y), 0, r)).astype(np.uint8)
    code[np.isnan(y)] = 127
    return code | (np.signbit(y).astype(np.uint8) << 7)


def write(codes, scales, x, row0):
    """x [n,Hkv,D] (float64) joins codes [Hkv,capacity,D] and scales [Hkv,capacity/64], in place."""
    n, Hkv, _ = x.shape
    for h in range(Hkv):
        for b in range(row0 // BLOCK, (row0 + n + BLOCK - 1) // BLOCK):
            lo, hi = max(row0, b * BLOCK), min(row0 + n, (b + 1) * BLOCK)
            new = x[lo - row0:hi - row0, h]
            s = scale_of(new)
            if lo > b * BLOCK:
                old = scales[h, b]
                s = max(s, old)
                if s != old:
                    codes[h, b * BLOCK:lo] = encode(VALUES[codes[h, b * BLOCK:lo]] * old, s)
            codes[h, lo:hi] = encode(new, s)
            scales[h, b] = s


def read(codes, scales, row0, rows):
    """[rows,Hkv,D] float64"""
    s = np.repeat(scales, BLOCK, axis=1)[:, row0:row0 + rows, None]
    return np.transpose(VALUES[codes[:, row0:row0 + rows]] * s, (1, 0, 2))
