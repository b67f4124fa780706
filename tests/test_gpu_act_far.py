"""Products with bias, activation and dropout, and their gradients, of tensors with more than 2^31 elements: rows at both ends and around each
2^31, 2^32 and 2^33 bytes or elements against the definition."""
import numpy as np
import pytest
import torch

import act_util as au
from test_gpu_act import OFFSET, SEED, TORCH, rng_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kept", [False, True])
def test_far_rows(dtype, kept):
    from paper_2401_11469_amd import zr
    rows, K, N, p = 530000, 8, 4104, 0.25
    g = torch.Generator(device="cuda").manual_seed(3)

    def rand(*shape):           # quarters of -2 .. 2: exact products and sums
        return (torch.randint(-8, 9, shape, generator=g, device="cuda", dtype=torch.int8).to(TORCH[dtype])) / 4

    X, W, b = rand(rows, K), rand(N, K), rand(N)
    keep = torch.arange(0, N, 3, dtype=torch.int32, device="cuda") if kept else None
    Y, Z = torch.empty(rows, N, dtype=TORCH[dtype], device="cuda"), torch.empty(rows, N, dtype=TORCH[dtype], device="cuda")
    how = dict(mode=zr.DROP_N, w_layout=zr.W_NK, act=zr.ACT_RELU, p=p, rng=rng_of())
    zr.resized_linear_act_fwd(X, W, keep, bias=b, Y=Y, Z=Z, **how)
    row32 = [(1 << e) // (N * es) for e in (31, 32, 33) for es in (1, 2, 4)]
    look = sorted({r for q in [0, *row32, rows - 3] for r in (q, q + 1, q + 2) if r < rows})
    at = torch.tensor(look, device="cuda")
    mask = torch.ones(N, device="cuda", dtype=torch.double)
    if kept:
        mask.zero_()[keep.long()] = 1
    z = X[at].double() @ W.double().t() * mask + b.double()
    factor = torch.from_numpy(np.concatenate([au.halves(SEED, OFFSET, 1, N, first_row=r) for r in look]) >= 16384).cuda().double() * (4 / 3)
    u = au.U[dtype] * (1 + 2.0 ** -10)
    assert ((Z[at].double() - z).abs() <= u * z.abs()).all()
    y = z.clamp(min=0) * factor
    assert ((Y[at].double() - y).abs() <= (u + 2 * au.F) * y).all()
    del Y
    v = rand(1, N)
    dY, dX = v.expand(rows, N).contiguous(), torch.empty_like(X)
    zr.resized_linear_act_bwd(X, W, dY, keep, Z=Z, dX=dX, need_dW=False, dgate=dY, **how)          # (dgate over dY)
    zz = Z[at].double()
    dg = v.double() * factor * zz.clamp(min=0)
    assert ((dY[at].double() - dg).abs() <= (u + 3 * au.F) * dg.abs()).all()
    dz = v.double() * factor * (zz > 0) * mask
    want, size = dz @ W.double(), dz.abs() @ W.double().abs()
    # (each dZ rounded to the type, at most N terms added in fp32)
    assert ((dX[at].double() - want).abs() <= u * want.abs() + ((u if dtype == "bf16" else 2 * au.F) + 64 * au.F) * size).all()
