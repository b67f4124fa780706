"""The backward join with some of its outputs wanted, where that decides how many workgroups share the rows: dx and dy have the same bits, a
call repeats its own, and every vector's gradient is within its bound."""
import numpy as np
import pytest
import torch

import act_util as au
from test_gpu_act import OFFSET, SEED, TORCH, rng_of, values, within

pytestmark = pytest.mark.gpu
VECTORS = ("bias", "gate", "post_w", "post_b", "pre_w", "pre_b")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", [au.RMS, au.LAYER])
@pytest.mark.parametrize("rows,cols", [(4099, 130), (5000, 768), (3600, 1024), (3600, 1100), (2000, 2100), (700, 4104)])
def test_any_outputs(rows, cols, kind, dtype):
    from paper_2401_11469_amd import zr
    g = np.random.default_rng(rows + cols)
    a = [values(g, dtype, rows, cols) for _ in range(4)]
    vec = {v: values(g, dtype, cols) for v in VECTORS}
    on_gpu = lambda v: torch.from_numpy(v).to(TORCH[dtype]).cuda()         # noqa: E731
    y, xo, d, dh = (on_gpu(v) for v in a)
    how = dict(norm=kind, post=True, pre=True, p=0.1, rng=rng_of(), scale=0.7, **{v: on_gpu(t) for v, t in vec.items() if v != "pre_b"})
    want = au.unjoin(a[2], a[3], a[1], a[0], kind, True, True, 1e-5, au.factor(SEED, OFFSET, rows, cols, 0.1), 0.7, vec, dtype)
    none = zr.block_join_bwd(d, dh, xo, y, **how)
    within(none[0].double().cpu().numpy(), *want["dx"], "dx")
    within(none[1].double().cpu().numpy(), *want["dy"], "dy")
    for some in (VECTORS, ("gate",), ("post_w", "pre_w"), ("bias",), ("post_b",), ("pre_b", "gate")):
        runs = []
        for _ in range(2):
            sums = {"d" + v: torch.empty(cols, dtype=TORCH[dtype], device="cuda") for v in some}
            dx, dy = zr.block_join_bwd(d, dh, xo, y, **how, **sums)
            assert torch.equal(dx, none[0]) and torch.equal(dy, none[1]), some
            runs.append(sums)
        for v in some:
            assert torch.equal(runs[0]["d" + v], runs[1]["d" + v]), (some, v)
            within(runs[0]["d" + v].double().cpu().numpy(), *want[v], f"d{v} of {some}")
