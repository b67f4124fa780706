"""Block-scaled values in 64 bits, from the definition, on the CPU: what the tests of these operators compare with.

A block of 32 values with a = max |x| has e = the smallest integer with a <= top * 2^e (within [-127, 127]); an element is the
grid value nearest to x * 2^-e, of two equally near ones the one with the even code.  NaN or infinity: the whole block is NaN.
"""
import numpy as np

E4M3, E2M1, INT8 = 0, 1, 2
NAMES = {E4M3: "e4m3", E2M1: "e2m1", INT8: "int8"}


def grid(fmt):
    """Non-negative values in the order of their codes."""
    if fmt == INT8:
        return np.arange(128) / 64.0
    if fmt == E2M1:
        return np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6.0])
    c = np.arange(127)
    return np.where(c < 8, (c & 7) * 2.0 ** -9, (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10.0))


def exponent(a, fmt):
    """The smallest e with a <= top 2^e, one number at a time, by trying."""
    top = grid(fmt)[-1]
    if a == 0:
        return -127
    e = int(np.floor(np.log2(a / top))) - 2
    while a > top * 2.0 ** e:
        e += 1
    return min(max(e, -127), 127)


def quantize(x, fmt):
    """x [rows, n] float64 -> (codes [rows, n] uint8, scale codes [rows, blocks] uint8, values [rows, n] float64)."""
    rows, n = x.shape
    nb = (n + 31) // 32
    g = grid(fmt)
    mids = (g[1:] + g[:-1]) / 2
    codes = np.zeros((rows, n), np.uint8)
    scales = np.zeros((rows, nb), np.uint8)
    vals = np.zeros((rows, n))
    for b in range(nb):
        s = slice(32 * b, min(n, 32 * b + 32))
        blk = x[:, s]
        bad = ~np.isfinite(blk).all(axis=1)
        safe = np.where(bad[:, None], 0.0, blk)
        e = np.array([exponent(a, fmt) for a in np.abs(safe).max(axis=1)])
        y = safe * 2.0 ** (-e.astype(float))[:, None]
        i = np.searchsorted(mids, np.abs(y))
        tie = (i < mids.size) & (mids[np.minimum(i, mids.size - 1)] == np.abs(y))
        i = i + (tie & (i % 2 == 1))
        v = np.where(np.signbit(y), -g[i], g[i])
        vals[:, s] = np.where(bad[:, None], np.nan, v * 2.0 ** e.astype(float)[:, None])
        if fmt == INT8:
            codes[:, s] = (v * 64).astype(np.int8).view(np.uint8)
        else:
            codes[:, s] = i | np.where(np.signbit(y), 8 if fmt == E2M1 else 128, 0)
        scales[:, b] = np.where(bad, 255, e + 127)
    return codes, scales, vals


def stored(codes, scales, fmt):
    """The bytes of the elements and of the scales, with their padding."""
    rows, n = codes.shape
    el = np.zeros((rows, (n + 127) // 128 * 128), np.uint8)
    el[:, :n] = codes
    if fmt == E2M1:
        el = el[:, 0::2] | (el[:, 1::2] << 4)
    sc = np.zeros((rows, (n + 511) // 512 * 16), np.uint8)
    for b in range(scales.shape[1]):
        sc[:, b // 16 * 16 + 4 * (b % 4) + b % 16 // 4] = scales[:, b]
    return el, sc
