"""Products of tiny and huge factors, whose products are of ordinary size, against float64.

Bounds: as in test_gpu_mx.py; for fp32 results with an 8-bit operand, which are multiplied in bf16, a factor below 2^-126 is off by half
of bf16's smallest step, 2^-134, so a result by 2^-134 times the sum of the other operand's magnitudes, and vice versa."""
import numpy as np
import pytest

from mx_util import E2M1, E4M3
from test_gpu_mx import U, mx_put, to_np
from test_gpu_mx import torch, zr  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("xf,wf", [(E4M3, E2M1), (E2M1, E2M1), (E4M3, E4M3)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N", [(4, 70), (40, 70), (1500, 2100)])
@pytest.mark.parametrize("ex,ew", [(-110, 90), (-124, 100), (-130, 110), (-134, 115), (110, -124), (115, -132), (-60, -58), (120, -118)])
def test_factors_at_the_ends_of_the_range(torch, zr, M, N, ex, ew, dtype, xf, wf):  # noqa: F811
    K = 100
    rng = np.random.Generator(np.random.PCG64(M + ex + 200))
    few = rng.standard_normal((8, K))                                       # (eight different rows and columns are enough)
    xm, xv = mx_put(torch, zr, few[rng.integers(0, 8, M)] * 2.0 ** ex, xf)
    wm, wv = mx_put(torch, zr, rng.standard_normal((8, K))[rng.integers(0, 8, N)] * 2.0 ** ew, wf)
    got = to_np(zr.mx_linear_fwd(xm, wm, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32))
    want = xv @ wv.T
    ax, aw = np.abs(xv), np.abs(wv)
    bound = (K + 8) * 2.0 ** -23 * (ax @ aw.T)
    if xf == E4M3 and dtype == "bf16":
        top = lambda v: np.pad(v, ((0, 0), (0, -K % 8))).reshape(v.shape[0], -1, 8).max(axis=2)  # noqa: E731
        bound += 2.0 ** -10 * (top(ax) @ top(aw).T)
    if xf == E4M3 and dtype == "f32":
        small = lambda v: (v < 2.0 ** -126) * 2.0 ** -134  # noqa: E731
        bound += small(ax) @ aw.T + ax @ small(aw).T + small(ax) @ small(aw).T
    bound = bound * (1 + U[dtype]) + U[dtype] * np.abs(want)
    bound += 2.0 ** -126                                                    # what may be taken for zero
    over = np.abs(got - want) - bound
    assert np.all(over <= 0), (int((over > 0).sum()), float(over.max()), float(np.abs(want).max()))
