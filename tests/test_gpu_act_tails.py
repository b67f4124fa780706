"""GELU of bf16 results where they are small: relative to the result, at every bf16 number of the range, in each kernel that computes it.

Bounds.  The tail T = Phi(-|z|) is off by 2.5e-4 of itself, its exponential (of z^2 / 2, from an argument that is off by 2 steps of fp32) by
(3 z^2 / 2 + 12) 2^-24 with the products around it, the result by half a step of bf16 (2^-8)."""
import numpy as np
import pytest
import torch
from scipy import special

import act_util as au

pytestmark = pytest.mark.gpu


def numbers():
    """Every bf16 number of [-13, -2^-12] and of [2^-12, 13]."""
    bits = np.arange(0x3980, 0x4151, dtype=np.uint32)
    z = (bits << 16).view(np.float32).astype(np.float64)
    assert z[0] == 2.0 ** -12 and z[-1] == 13.0
    return np.concatenate([-z, z])


def expected(z):
    """(value, its bound), (slope, its bound)"""
    cdf, T, phi = special.ndtr(z), special.ndtr(-abs(z)), np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
    rel, u = (1.5 * z * z + 12) * au.F, au.U["bf16"] * (1 + 2.0 ** -10)
    a, s = z * cdf, cdf + z * phi
    # (of max(z, 0) - |z| T the error of T counts as |z| T; of the slope's two terms each its own)
    return ((a, u * abs(a) + 2.5e-4 * abs(z) * T + rel * (abs(z) * T + abs(a)) + 1e-37),
            (s, u * abs(s) + 2.5e-4 * T + rel * (abs(z) * phi + T + cdf) + 1e-37))


def check(got, want, bound, z, name):
    bad = ~(abs(got - want) <= bound)
    assert not bad.any(), (name, z[bad][:5], got[bad][:5], want[bad][:5], (abs(got - want) / bound).max())


@pytest.mark.parametrize("M,kn", [(1, True), (1, False), (16, True), (40, True), (40, False), (200, True)])
def test_values(M, kn):
    """Through a product with one column of ones, whose sums are the numbers."""
    from paper_2401_11469_amd import zr
    z = numbers()
    t = torch.from_numpy(z).bfloat16().cuda()
    K = 64
    W = torch.zeros(K, len(z), dtype=torch.bfloat16, device="cuda")
    W[0] = t
    X = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    X[:, 0] = 1
    Y = zr.resized_linear_act_fwd(X, W if kn else W.t().contiguous(), act=zr.ACT_GELU, w_layout=zr.W_KN if kn else zr.W_NK)
    assert (Y == Y[0]).all()
    check(Y[0].double().cpu().numpy(), *expected(z)[0], z, "value")


def test_values_on_large_tiles():
    from paper_2401_11469_amd import zr
    z = np.tile(numbers(), 3)[:8192]
    W = torch.zeros(8192, 64, dtype=torch.bfloat16, device="cuda")
    W[:, 0] = torch.from_numpy(z).bfloat16()
    X = torch.zeros(2304, 64, dtype=torch.bfloat16, device="cuda")
    X[:, 0] = 1
    Y = zr.resized_linear_act_fwd(X, W, act=zr.ACT_GELU, w_layout=zr.W_NK)
    assert (Y == Y[0]).all()
    check(Y[0].double().cpu().numpy(), *expected(z)[0], z, "value")


@pytest.mark.parametrize("kept", [False, True])
def test_slopes_and_gate_gradients(kept):
    """dY of ones and an identity for W: dX holds dZ, dgate the values."""
    from paper_2401_11469_amd import zr
    z = numbers()
    n = 960
    parts = [np.resize(z[i:i + n], n) for i in range(0, len(z), n)]
    Z = torch.from_numpy(np.stack(parts)).bfloat16().cuda()
    keep = torch.arange(0, n, 3, dtype=torch.int32, device="cuda") if kept else None
    dg = torch.empty_like(Z)
    dX, _ = zr.resized_linear_act_bwd(None, torch.eye(n, dtype=torch.bfloat16, device="cuda"), torch.ones_like(Z), keep, mode=zr.DROP_N, act=zr.ACT_GELU, Z=Z,
                                      dgate=dg, need_dW=False)
    z = np.stack(parts)
    (a, ea), (s, es) = expected(z)
    check(dg.double().cpu().numpy(), a, ea, z, "dgate")
    got = dX.double().cpu().numpy()
    if kept:
        mask = np.zeros(n, dtype=bool)
        mask[::3] = True
        assert (got[:, ~mask] == 0).all()
        got, s, es, z = got[:, mask], s[:, mask], es[:, mask], z[:, mask]
    check(got, s, es, z, "slope")
