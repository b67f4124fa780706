"""The bounds of act_bounds.py on the CPU: the kernels' formulas in fp32 keep them, and results that only an absolute bound lets pass do not."""
import numpy as np
import pytest
from scipy import special

import act_util as au
from act_bounds import bounds, points
from test_act_tail_formula import constants

f32 = np.float32


def sigmoid(x):
    with np.errstate(over="ignore"):
        return (f32(1) / (f32(1) + np.exp(-x, dtype=f32))).astype(f32)


def formula(kind, z):
    """Value and slope as the fp32 kernels compute them (their exponentials and erfc by numpy's, rounded once)."""
    z = z.astype(f32)
    with np.errstate(over="ignore", under="ignore", invalid="ignore"):
        if kind == au.GELU:
            cdf = f32(0.5) * special.erfc((f32(-0.70710678) * z).astype(np.float64)).astype(f32)
            return z * cdf, z * (f32(0.39894228) * np.exp(f32(-0.5) * z * z, dtype=f32)) + cdf
        if kind == au.SILU:
            t = sigmoid(z)
            return z * t, t * (z * (1 - t) + 1)
        zz = z * z
        t = sigmoid(f32(1.59576912) * z * (f32(0.044715) * zz + 1))
        return z * t, z * t * (1 - t) * (f32(1.59576912) * (f32(0.134145) * np.minimum(zz, f32(1e12)) + 1)) + t


@pytest.mark.parametrize("kind", [au.GELU, au.GELU_TANH, au.SILU])
def test_formulas_in_fp32_keep_the_bounds(kind):
    z = points("f32")
    (a, ea), (s, es) = bounds(kind, z, "f32")
    va, vs = formula(kind, z)
    assert (abs(va - a) <= ea).all() and (abs(vs - s) <= es).all(), ((abs(va - a) / ea).max(), (abs(vs - s) / es).max())


def test_bf16_formula_is_too_coarse_for_fp32_results():
    slope, c = constants()
    z = points("f32")
    z = z[abs(z) < 13]
    t = 1 / (1 + slope * abs(z))
    tail = np.polyval(c, t) * t * np.exp(-z * z / 2)
    (a, ea), (s, es) = bounds(au.GELU, z, "f32")
    assert (abs(np.maximum(z, 0) - abs(z) * tail - a) > ea).sum() > len(z) / 20
    (_, eb), _ = bounds(au.GELU, z, "bf16")
    assert (abs(np.maximum(z, 0) - abs(z) * tail - a) <= eb).all()
    # formula 7.1.26 of Abramowitz and Stegun bounds its error absolutely: more than a bf16 result may be off, half a step of bf16 included, from -9 to -12
    t = 1 / (1 + 0.3275911 * np.sqrt(0.5) * abs(z))
    tail = 0.5 * np.polyval([1.061405429, -1.453152027, 1.421413741, -0.284496736, 0.254829592], t) * t * np.exp(-z * z / 2)
    off = abs(np.maximum(z, 0) - abs(z) * tail - a)
    assert (off > 3 * ea)[(z < -7) & (z > -12)].all() and (off > eb)[(z < -9) & (z > -12)].all()


@pytest.mark.parametrize("kind", [au.GELU, au.GELU_TANH, au.SILU])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nothing_passes_for_a_small_result(kind, dtype):
    """0 in place of a small value, or a step of the type too much, is refused down to 2^-110."""
    z = points(dtype)
    (a, ea), (s, es) = bounds(kind, z, dtype)
    small = (abs(a) > 2.0 ** -110) & (z < 0)
    assert small.sum() > 1000 and (ea[small] < 0.01 * abs(a[small])).all()
    # (the slope's zero near -1.3 or -0.75 is the difference of two terms)
    low = (abs(s) > 2.0 ** -110) & (z < -3)
    assert low.sum() > 100 and (es[low] < 0.02 * abs(s[low])).all()
