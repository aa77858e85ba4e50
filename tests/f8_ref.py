"""Plain reference of 8-bit storage (blocks of 128 elements of a row, e4m3 codes
and a power-of-two scale each), in numpy and 64 bits; shares nothing with the
kernels."""
import math

import numpy as np

BLOCK = 128


def code_values():
    """The value of every e4m3 byte (1 sign, 4 exponent bits biased by 7, 3
    mantissa bits; 0x7F and 0xFF are NaN, there is no infinity)."""
    v = np.zeros(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        mag = math.ldexp(8 + m, e - 10) if e else math.ldexp(m, -9)
        v[b] = math.nan if (b & 127) == 127 else (-mag if b & 128 else mag)
    return v


VALUES = code_values()
_POSITIVE = VALUES[:127]


def quantize(w):
    """(codes, scales) of a float32 matrix, by search: the nearest value, of two
    equally near ones that with the even code."""
    w = np.asarray(w, dtype=np.float32).astype(np.float64)
    rows, cols = w.shape
    blocks = -(-cols // BLOCK)
    codes = np.zeros((rows, blocks * BLOCK), dtype=np.uint8)
    scales = np.zeros((rows, -(-blocks // 4) * 4), dtype=np.uint8)
    for r in range(rows):
        for b in range(blocks):
            part = w[r, b * BLOCK:(b + 1) * BLOCK]
            fin = np.abs(part[np.isfinite(part)])
            top = float(fin.max()) if fin.size else 0.0
            e = 0
            if top > 0:
                e = -127
                while top > 448.0 * 2.0 ** e:
                    e += 1
            x = np.where(np.isfinite(part), np.abs(part), 0.0) / 2.0 ** e
            hi = np.clip(np.searchsorted(_POSITIVE, x), 0, 126)
            lo = np.maximum(hi - 1, 0)
            dl, dh = x - _POSITIVE[lo], _POSITIVE[hi] - x
            c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
            c = np.where(np.signbit(part), c + 128, c)
            codes[r, b * BLOCK:b * BLOCK + part.size] = np.where(np.isfinite(part), c, 127)
            scales[r, b] = e + 127
    return codes, scales


def dequantize(codes, scales, cols):
    blocks = -(-cols // BLOCK)
    s = np.exp2(scales[:, :blocks].astype(np.float64) - 127)
    return (VALUES[codes] * np.repeat(s, BLOCK, axis=1))[:, :cols]
