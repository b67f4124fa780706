"""How far the activations and their slopes may be off for an exact argument: relative to the value, in each type by its own roundings.

f = 2^-24, half a step of fp32 relative to the value; u: the same of the result's type.
 * An exponential of an argument of size w that is off by k f w is off by (k w + 3) f of itself.  SiLU: w = |z|, from one product (bf16) or none.
   GELU: w = z^2 / 2, from two products and a constant (in erfc the argument's error counts z^2 + 1 times).  Its tanh form:
   w = 1.6 |z| + 0.072 |z|^3, from four products, a sum and two constants.  k = 7 covers each.
 * What is made of it takes at most 9 f more: a sum with 1, a reciprocal or the library's erfc (4 steps), two products.
 * bf16 results of GELU take a formula for the tail T = Phi(-|z|) that is off by 2.5e-4 of T; the value is max(z, 0) - |z| T.
 * The sigmoid t goes into slopes as 1 - t as well, which is off by 3 f besides.
 * A sigmoid below 2^-126 may come out as 0."""
import numpy as np
from scipy import special

import act_util as au

TINY = 2.0 ** -126


def bounds(kind, z, dtype):
    """(value, its bound), (slope, its bound)"""
    f, u = au.F, au.U[dtype] * (1 + 2.0 ** -10)
    z = np.asarray(z, dtype=np.float64)
    n = abs(z)
    with np.errstate(over="ignore", under="ignore", invalid="ignore"):
        a, s = au.act(kind, z)
        if kind in (au.NONE, au.RELU):
            return (a, 0 * z), (s, 0 * z)
        if kind == au.GELU:
            rel = (3.5 * z * z + 12) * f
            cdf, T, phi = special.ndtr(z), special.ndtr(-n), np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
            if dtype == "bf16":
                ea, es = (2.5e-4 + rel) * n * T + 3 * f * abs(a), (2.5e-4 + rel) * T + rel * n * phi + 3 * f * cdf
            else:
                ea, es = rel * abs(a), rel * (cdf + n * phi)
            return (a, ea + u * abs(a) + n * TINY), (s, es + u * abs(s) + (1 + n) * TINY)
        w = n if kind == au.SILU else 1.6 * n + 0.072 * n ** 3
        x = z if kind == au.SILU else 2 * np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)
        t, rest = special.expit(x), special.expit(-x)
        D = 1.0 if kind == au.SILU else 1.5958 * (1 + 0.134145 * np.minimum(z * z, 1e12))
        rel = (7 * np.minimum(w, 1e4) + 12) * f
        # (the sigmoid is off by rel of itself where it is small, by rel (1 - t) and a rounding where it is not)
        et = rel * t * rest + 3 * f * t + TINY
        es = et * (1 + n * D * rest) + n * t * D * (rel * t * rest + 3 * f) + 9 * f * (t + n * t * rest * D)
        # (past 40 both are what they tend to: nothing is left of 1 - t but a rounding, of which z t (1 - t) makes nothing)
        es = np.where(w > 100, 4 * f * t + (1 + n) * TINY, es)
        return (a, n * et + u * abs(a) + f * abs(a)), (s, es + u * abs(s))


def points(dtype):
    """Arguments of every size: bf16 all numbers of 2^-12 to 128 and their negatives; fp32 as many spread over the same, and large ones of both."""
    if dtype == "bf16":
        bits = np.arange(0x3980, 0x4301, dtype=np.uint32)
        z = (bits << 16).view(np.float32).astype(np.float64)
    else:
        g = np.random.default_rng(12)
        z = np.concatenate([2.0 ** g.uniform(-12, 7, 2500), g.uniform(0, 14, 1500)]).astype(np.float32).astype(np.float64)
    z = np.concatenate([z, [0.0, 2.0 ** -100, 256.0, 1024.0, 2.0 ** 20, 2.0 ** 40]])
    return np.concatenate([z, -z])
