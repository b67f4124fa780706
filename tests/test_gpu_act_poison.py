"""NaN where nothing is to be read as a value: pruned columns of X and slices of W, the pitch behind every row, memory beside the tensors, and the
workspace.  Every result has the same bits as with numbers there."""
import numpy as np
import pytest
import torch

import act_util as au
from test_gpu_act import TORCH, keep_of, rng_of, values

pytestmark = pytest.mark.gpu


def placed(a, dtype, pad, off, fill):
    """The matrix with `pad` elements behind each row, `off` before the first, all of them `fill`."""
    rows, cols = a.shape
    buf = torch.full((off + (rows + 2) * (cols + pad) + 64,), fill, dtype=TORCH[dtype], device="cuda")
    t = buf[off + cols + pad:off + cols + pad + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    t.copy_(a)
    return t


SIZES = [(1, 64, 40, 0.25, 0, 0), (3, 136, 520, 0.4, 8, 0), (8, 1000, 264, 0.25, 0, 0), (16, 77, 129, 0.3, 3, 1), (40, 136, 120, 0.3, 8, 8),
         (200, 328, 264, 0.25, 0, 0), (257, 130, 515, 0.4, 1, 3), (1024, 192, 1280, 0.25, 0, 0), (300, 40, 333, 0.9, 0, 0)]
LARGE = [(2304, 328, 4000, 0.5, 8, 0), (4096, 96, 2064, 0.95, 0, 0)]          # (for the large tiles, which are those of bf16)


@pytest.mark.parametrize("mode_k,kn", [(0, 0), (0, 1), (1, 0), (1, 1)])
@pytest.mark.parametrize("M,K,N,ratio,pad,off,dtype", [(*s, "bf16") for s in SIZES + LARGE] + [(*s, "f32") for s in SIZES])
def test_products(M, K, N, ratio, pad, off, mode_k, kn, dtype):
    from paper_2401_11469_amd import zr
    g = np.random.default_rng(M + K + N)
    n = K if mode_k else N
    kept = keep_of(g, n, ratio)
    keep = torch.from_numpy(kept.astype(np.int32)).cuda()
    pruned = torch.ones(n, dtype=torch.bool)
    pruned[kept] = False
    X, W, G, R, Z, dY = (torch.from_numpy(values(g, dtype, *s)) for s in ((M, K), (K, N), (M, N), (M, N), (M, N), (M, N)))
    b = torch.from_numpy(values(g, dtype, N)).to(TORCH[dtype]).cuda()
    mode, layout = (zr.DROP_K if mode_k else zr.DROP_N), (zr.W_KN if kn else zr.W_NK)
    results = []
    for bad in (1.0, float("nan")):
        x, w = X.clone(), W.clone()
        if mode_k:
            x[:, pruned] = bad
            w[pruned] = bad
        else:
            w[:, pruned] = bad
        at = {k: placed(t, dtype, pad, off, bad) for k, t in (("X", x), ("W", w if kn else w.t()), ("G", G), ("R", R), ("Z", Z), ("dY", dY))}
        out = {k: placed(torch.full(s, bad), dtype, pad, off, bad) for k, s in (("Y", (M, N)), ("Zo", (M, N)), ("dX", (M, K)), ("dW", (K, N) if kn else (N, K)), ("dG", (M, N)))}
        how = dict(mode=mode, act=au.SILU, gate=at["G"], p=0.1, rng=rng_of(), w_layout=layout)
        for backward in (False, True):
            ws = torch.full((zr.act_workspace_bytes(M, K, N, len(kept), mode, TORCH[dtype], backward) // 4 + 4,), bad, device="cuda").view(torch.uint8)
            if backward:
                db = torch.full((N,), bad, dtype=TORCH[dtype], device="cuda")
                zr.resized_linear_act_bwd(at["X"], at["W"], at["dY"], keep, Z=at["Z"], dX=out["dX"], dW=out["dW"], dbias=db, dgate=out["dG"], workspace=ws, **how)
            else:
                zr.resized_linear_act_fwd(at["X"], at["W"], keep, bias=b, residual=at["R"], Y=out["Y"], Z=out["Zo"], workspace=ws, **how)
        small = zr.resized_linear_act_fwd(at["X"], at["W"], keep, bias=b, residual=at["R"], **how)
        results.append([*out.values(), db, small])
    for a, c in zip(*results):
        assert a.isfinite().all() and torch.equal(a, c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pad,off", [(1, 5, 3, 1), (7, 40, 0, 0), (13, 513, 1, 0), (300, 1023, 2, 3), (9, 2000, 8, 0), (5, 4100, 0, 1), (6, 5121, 7, 0), (3, 9001, 1, 1)])
@pytest.mark.parametrize("kind", [au.RMS, au.LAYER])
def test_joins(rows, cols, pad, off, kind, dtype):
    from paper_2401_11469_amd import zr
    g = np.random.default_rng(rows + cols)
    Y, X, D, H = (torch.from_numpy(values(g, dtype, rows, cols)) for _ in range(4))
    names = ("bias", "gate", "post_w", "post_b", "pre_w", "pre_b")
    vectors = {v: torch.from_numpy(values(g, dtype, cols)) for v in names}
    results = []
    for bad in (1.0, float("nan")):
        y, x, d, h = (placed(t, dtype, pad, off, bad) for t in (Y, X, D, H))
        xo, ho, dx, dy = (placed(torch.full((rows, cols), bad), dtype, pad, off, bad) for _ in range(4))
        vec = {v: placed(t[None], dtype, 0, off, bad)[0] for v, t in vectors.items()}
        how = dict(norm=kind, post=True, pre=True, p=0.1, rng=rng_of(), scale=0.7)
        zr.block_join_fwd(y, x, x_out=xo, h=ho, **how, **vec)
        sums = {"d" + v: placed(torch.full((1, cols), bad), dtype, 0, off, bad)[0] for v in names}
        ws = torch.full((zr.block_join_workspace_bytes(rows, cols) // 4,), bad, device="cuda").view(torch.uint8)
        vec.pop("pre_b")
        zr.block_join_bwd(d, h, xo, y, dx=dx, dy=dy, workspace=ws, **how, **vec, **sums)
        results.append([xo, ho, dx, dy, *sums.values()])
    for a, c in zip(*results):
        assert a.isfinite().all() and torch.equal(a, c)
