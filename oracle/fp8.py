"""8-bit floating point with one scale for each block of 128 (oracle; test
infrastructure only): OCP E4M3 and E5M2 by their tables of values, block and
tile quantization, and the words of the dropout mask.

The tables are built from the definition (sign, exponent, fraction) and a
value is encoded by searching the midpoints of neighbouring codes, ties to the
even code, in float64.
"""

import numpy as np

from . import philox

BLOCK = 128
# exponent bits, fraction bits, bias, codes of finite magnitudes
_SHAPES = {"e4m3": (4, 3, 7, 0x7F), "e5m2": (5, 2, 15, 0x7C)}
TOP = {"e4m3": 448.0, "e5m2": 57344.0}


def values(fmt):
    """Magnitudes of the finite codes 0, 1, ..., ascending."""
    _, m, bias, n = _SHAPES[fmt]
    out = np.empty(n)
    for c in range(n):
        e, f = c >> m, c & ((1 << m) - 1)
        out[c] = f * 2.0 ** (1 - bias - m) if e == 0 else (1 + f / 2.0 ** m) * 2.0 ** (e - bias)
    return out


def decode(codes, fmt):
    """float64 values of code bytes; the codes past the finite ones give NaN
    (E5M2's infinities included: no quantizer here writes one)."""
    t = values(fmt)
    c = np.asarray(codes, np.uint8)
    mag = c & 0x7F
    v = np.where(mag < t.size, t[np.minimum(mag, t.size - 1)], np.nan)
    return np.where(c & 0x80, -v, v)


def encode(y, fmt):
    """Code bytes of float64 ``y``: nearest, ties to the even code, saturating;
    NaN gives 0xFF (a NaN of both formats)."""
    t = values(fmt)
    mid = (t[1:] + t[:-1]) / 2
    a = np.abs(np.asarray(y, np.float64))
    a = np.where(np.isnan(a), 0.0, a)
    lo, hi = np.searchsorted(mid, a, "left"), np.searchsorted(mid, a, "right")
    code = np.where(lo != hi, np.where(lo % 2 == 0, lo, hi), lo).astype(np.uint8)
    code |= np.where(np.signbit(y), 0x80, 0).astype(np.uint8)
    return np.where(np.isnan(y), np.uint8(0xFF), code).astype(np.uint8)


def block_scale(a, fmt, scale):
    """(divisor over F, scale held) of block maxima ``a``, float64."""
    a, top = np.asarray(a, np.float64), TOP[fmt]
    if scale == "e8m0":
        m, e = np.frexp(np.where(a > 0, a, top))     # a / F = m / (1.75/2) 2^(...): compare fractions
        _, et = np.frexp(top)
        p = np.exp2(np.maximum(e - et + (m > 0.875), -126.0))
        p = np.where(a > 0, p, 1.0)
        return p * top, p
    ae = np.where(a > 0, np.maximum(a, top * 2.0 ** -126), top)
    return ae, (ae.astype(np.float32) / np.float32(top)).astype(np.float64)


def _quantize(v, a, fmt, scale):
    """Codes of ``v`` and held scales, for block maxima ``a`` that broadcast."""
    d, s = block_scale(a, fmt, scale)
    y = np.where(np.isfinite(v), np.where(np.isfinite(v), v, 0.0) * TOP[fmt] / d, np.nan)
    return encode(np.where(np.isnan(y), np.nan, np.where(y == 0, np.copysign(0.0, v), y)), fmt), s


def quantize_rows(x, fmt, scale):
    """x [R, C] (float64) along its rows: codes [R, pad(C)], scales [pad(C) / 128, R]."""
    R, C = x.shape
    v = np.pad(np.asarray(x, np.float64), ((0, 0), (0, -C % BLOCK))).reshape(R, -1, BLOCK)
    a = np.where(np.isfinite(v), np.abs(v), 0.0).max(2, keepdims=True) if v.size else np.zeros((*v.shape[:2], 1))
    q, s = _quantize(v, a, fmt, scale)
    return q.reshape(R, -1), s[:, :, 0].T


def quantize_tiles(w, scale):
    """w [R, C] in 128 x 128 tiles, E4M3: codes [R, pad(C)], scales [pad(R) / 128, pad(C) / 128]."""
    R, C = w.shape
    v = np.pad(np.asarray(w, np.float64), ((0, -R % BLOCK), (0, -C % BLOCK)))
    t = v.reshape(v.shape[0] // BLOCK, BLOCK, v.shape[1] // BLOCK, BLOCK)
    a = np.where(np.isfinite(t), np.abs(t), 0.0).max((1, 3), keepdims=True)
    q, s = _quantize(t, a, "e4m3", scale)
    return q.reshape(v.shape)[:R], s[:, 0, :, 0]


def decoded_rows(codes, scales, fmt):
    """float64 values [R, pad(C)] of a row quantization."""
    R = codes.shape[0]
    return (decode(codes, fmt).reshape(R, -1, BLOCK) * scales.T[:, :, None]).reshape(R, -1)


def decoded_tiles(codes, scales):
    R = codes.shape[0]
    s = np.repeat(np.repeat(scales, BLOCK, 0)[:R], BLOCK, 1)
    return decode(codes, "e4m3") * s


def dropout_words(seed, tensor_id, index):
    """The 16 bits of each element index: word (i % 8) / 2, half i % 2, of
    Philox4x32-10 at counter (i / 8, tensor id, 1)."""
    i = np.asarray(index, np.int64)
    uj, inv = np.unique(i >> 3, return_inverse=True)
    j = uj.astype(np.uint64)
    ctr = np.stack([j & philox.MASK, j >> np.uint64(32), np.full_like(j, np.uint64(tensor_id & 0xFFFFFFFF)),
                    np.ones_like(j)], axis=-1)
    seed = int(seed) & 0xFFFFFFFFFFFFFFFF
    w = philox.philox4x32_10(ctr, (seed & 0xFFFFFFFF, seed >> 32))
    e = i & 7
    return (w[inv.reshape(i.shape), e >> 1] >> (16 * (e & 1)).astype(np.uint32)) & np.uint32(0xFFFF)
