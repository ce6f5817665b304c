"""The 8-bit format of a layer's products in numpy, from its definition (float64 throughout)."""
import numpy as np

BLOCK = 128

# the 256 codes' values: sign, 4 exponent bits (bias 7, 0: subnormal), 3 mantissa bits; 0x7f and 0xff are NaN
_U = np.arange(256)
_F, _M = (_U >> 3) & 15, _U & 7
CODE_VALUES = np.where(_F > 0, (8.0 + _M) * 2.0 ** (_F - 10.0), _M * 2.0 ** -9) * np.where(_U > 127, -1.0, 1.0)
CODE_VALUES[[0x7F, 0xFF]] = np.nan


def scale_width(K):
    return 4 * -(-K // 512)


def _amax(x, rows):
    M, K = x.shape
    p = np.zeros((-(-M // rows) * rows, -(-K // BLOCK) * BLOCK))
    p[:M, :K] = np.abs(x)  # a NaN stays one
    return p.reshape(-1, rows, p.shape[1] // BLOCK, BLOCK).max((1, 3))


def scale_bytes(x, rows):
    """[ceil(M / rows), scale_width(K)]"""
    a = _amax(x, rows)
    with np.errstate(invalid="ignore"):
        m, e = np.frexp(np.where(np.isfinite(a), a, 1.0))
    e = np.clip(np.where(a > 0, e - 9 + (m > 0.875), -1000), -117, 119)  # 448 = 0.875 * 2^9
    b = np.where(np.isfinite(a), e + 127, 255).astype(np.uint8)
    out = np.zeros((b.shape[0], scale_width(x.shape[1])), np.uint8)
    out[:, : b.shape[1]] = b
    return out


def scales(b, M, K, rows):
    """float64 [M, K] of scale bytes"""
    s = np.where(b == 255, np.nan, np.exp2(b.astype(np.float64) - 127))
    return np.repeat(np.repeat(s, rows, 0)[:M], BLOCK, 1)[:, :K]


def codes(x, rows):
    """code bytes [M, K]: the nearest of the format's values, ties to the even code"""
    s = scales(scale_bytes(x, rows), *x.shape, rows)
    bad = np.isnan(s)
    v = np.where(bad, 0.0, x / np.where(bad, 1.0, s))
    size = np.minimum(np.abs(v), 448.0)
    pos = CODE_VALUES[:127]
    i = np.clip(np.searchsorted(pos, size, side="right") - 1, 0, 125)
    low, high = pos[i], pos[i + 1]
    up = (size - low > high - size) | ((size - low == high - size) & (i % 2 == 1))
    c = i + up
    return np.where(bad, 0, c + np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def values(c, b, rows):
    """float64 [M, K] that codes and scale bytes stand for"""
    return CODE_VALUES[c] * scales(b, *c.shape, rows)
