"""The gradients of a product with dropout: what gate, Z and dY hold at a dropped place reaches none of them, as it reaches no output of the
forward pass."""
import numpy as np
import pytest
import torch

import act_util as au
from test_gpu_act import OFFSET, SEED, TORCH, keep_of, rng_of, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mode_k,M,K,N,ratio", [(0, 24, 40, 72, 0.0), (0, 150, 64, 600, 0.25), (1, 33, 96, 77, 0.3), (0, 7, 40, 1100, 0.5), (1, 300, 72, 264, 0.0)])
def test_dropped_places_hold_anything(mode_k, M, K, N, ratio, act, dtype):
    from paper_2401_11469_amd import zr
    g = np.random.default_rng(M + N)
    f = au.factor(SEED, OFFSET, M, N, 0.5)
    dropped = torch.from_numpy(f == 0).cuda()
    X, W, Z, G, dY = (torch.from_numpy(values(g, dtype, *s)).to(TORCH[dtype]).cuda() for s in ((M, K), (K, N), (M, N), (M, N), (M, N)))
    n = K if mode_k else N
    keep = torch.from_numpy(keep_of(g, n, ratio).astype(np.int32)).cuda() if ratio else None

    def back(Z, G, dY):
        db, dG = torch.empty(N, dtype=TORCH[dtype], device="cuda"), torch.empty_like(Z)
        dX, dW = zr.resized_linear_act_bwd(X, W, dY, keep, mode=zr.DROP_K if mode_k else zr.DROP_N, act=act, Z=Z, gate=G, p=0.5, rng=rng_of(), dbias=db, dgate=dG)
        return dX, dW, db, dG

    want = back(Z, G, dY)
    assert all(t.isfinite().all() for t in want) and (want[3][dropped] == 0).all()
    for bad in (float("nan"), float("inf"), -float("inf"), 3e38):
        spoiled = lambda t: torch.where(dropped, torch.full_like(t, bad), t)         # noqa: E731
        for args in ((spoiled(Z), G, dY), (Z, spoiled(G), dY), (Z, G, spoiled(dY)), (spoiled(Z), spoiled(G), spoiled(dY))):
            for got, t, name in zip(back(*args), want, ("dX", "dW", "dbias", "dgate")):
                assert torch.equal(got, t), (name, bad)
