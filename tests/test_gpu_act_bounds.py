"""Activations and their slopes on the GPU, relative to the value, with the bounds of act_bounds.py: every kind and type, in each kernel."""
import numpy as np
import pytest
import torch

import act_util as au
from act_bounds import bounds, points
from test_gpu_act import TORCH

pytestmark = pytest.mark.gpu


def check(got, want, bound, z, name):
    got = got.double().cpu().numpy()
    bad = ~(abs(got - want) <= bound)
    assert not bad.any(), (name, int(bad.sum()), z[bad][:4], got[bad][:4], want[bad][:4], np.nanmax(abs(got - want) / bound))


@pytest.mark.parametrize("kind", [au.RELU, au.GELU, au.GELU_TANH, au.SILU])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,kn", [(1, True), (1, False), (40, True), (300, False)])
def test_values(kind, dtype, M, kn):
    """Through a product with one column of ones: its sums are the arguments."""
    from paper_2401_11469_amd import zr
    z = points(dtype)
    W = torch.zeros(64, len(z), dtype=TORCH[dtype], device="cuda")
    W[0] = torch.from_numpy(z).to(TORCH[dtype])
    X = torch.zeros(M, 64, dtype=TORCH[dtype], device="cuda")
    X[:, 0] = 1
    Y = zr.resized_linear_act_fwd(X, W if kn else W.t().contiguous(), act=kind, w_layout=zr.W_KN if kn else zr.W_NK)
    assert (Y == Y[0]).all()
    check(Y[0], *bounds(kind, z, dtype)[0], z, "value")


@pytest.mark.parametrize("kind", [au.RELU, au.GELU, au.GELU_TANH, au.SILU])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kept", [False, True])
def test_slopes_and_gate_gradients(kind, dtype, kept):
    """dY of ones and an identity for W: dX holds dZ, dgate the values."""
    from paper_2401_11469_amd import zr
    z, n = points(dtype), 960
    z = np.stack([np.resize(z[i:i + n], n) for i in range(0, len(z), n)])
    Z = torch.from_numpy(z).to(TORCH[dtype]).cuda()
    some = np.arange(0, n, 3) if kept else np.arange(n)
    keep = torch.from_numpy(some.astype(np.int32)).cuda() if kept else None
    dg = torch.empty_like(Z)
    dX, _ = zr.resized_linear_act_bwd(None, torch.eye(n, dtype=TORCH[dtype], device="cuda"), torch.ones_like(Z), keep, mode=zr.DROP_N, act=kind, Z=Z,
                                      dgate=dg, need_dW=False)
    (a, ea), (s, es) = bounds(kind, z, dtype)
    check(dg, a, ea, z, "dgate")
    check(dX[:, some], s[:, some], es[:, some], z[:, some], "slope")
