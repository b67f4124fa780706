"""The backward join where a workgroup takes several rows at a time and their number is no multiple of that: the threads behind the last row
add nothing to the vectors' gradients, whatever the last row holds at its dropped places."""
import numpy as np
import pytest
import torch

import act_util as au
from test_gpu_act import OFFSET, SEED, TORCH, rng_of, values

pytestmark = pytest.mark.gpu


def back(y, xo, d, dh, vec, kind, post, pre, p, rng, eps=1e-5):
    from paper_2401_11469_amd import zr
    names = [v for v in ("bias", "gate", "post_w", "post_b", "pre_w", "pre_b") if not (v[:4] == "post" and not post or v[:3] == "pre" and not pre)]
    sums = {"d" + v: torch.full_like(d[0], 77.0) for v in names}
    use = {v: t for v, t in vec.items() if v in names and v != "pre_b"}
    dx, dy = zr.block_join_bwd(d, dh if pre else None, xo if pre else None, y, norm=kind, post=post, pre=pre, p=p, rng=rng, eps=eps, **use, **sums)
    return dict(dx=dx, dy=dy, **sums)


@pytest.mark.parametrize("post,pre", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("kind", [au.RMS, au.LAYER])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 96), (5, 40), (7, 512), (9, 700), (4099, 130), (1801, 1024)])
def test_dropped_places_of_the_last_row_hold_anything(rows, cols, dtype, kind, post, pre):
    g = np.random.default_rng(rows + cols)
    y, xo, d, dh = (torch.from_numpy(values(g, dtype, rows, cols)).to(TORCH[dtype]).cuda() for _ in range(4))
    vec = {v: torch.from_numpy(values(g, dtype, cols)).to(TORCH[dtype]).cuda() for v in ("bias", "gate", "post_w", "post_b", "pre_w")}
    dropped = torch.from_numpy(au.factor(SEED, OFFSET, rows, cols, 0.5) == 0).cuda()
    want = back(torch.where(dropped, 0, y), xo, d, dh, vec, kind, post, pre, 0.5, rng_of())
    for name, t in want.items():
        assert t.isfinite().all(), name
    for bad in (float("nan"), float("inf"), 3e38):
        got = back(torch.where(dropped, bad, y.float()).to(y.dtype), xo, d, dh, vec, kind, post, pre, 0.5, rng_of())
        for name, t in want.items():
            assert torch.equal(got[name], t), (name, bad)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("post,pre", [(True, False), (True, True)])
def test_a_row_behind_the_last_that_is_dropped_as_a_whole(dtype, post, pre):
    """Root mean square of zeros with eps 0 has no value; no such row is there, although the draws of the next one would make it."""
    rows, cols, p = 5, 2, 0.5
    offset = next(o for o in range(1000) if au.factor(SEED, o, rows, cols, p).any(axis=1).all() and not au.factor(SEED, o, rows + 1, cols, p)[rows].any())
    g = np.random.default_rng(3)
    y, xo, d, dh = (torch.from_numpy(values(g, dtype, rows, cols)).to(TORCH[dtype]).cuda() for _ in range(4))
    got = back(y, xo, d, dh, {}, au.RMS, post, pre, p, rng_of(SEED, offset), eps=0.0)
    for name, t in got.items():
        assert t.isfinite().all(), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_gate_that_is_no_number_stays_in_its_column(dtype):
    """An infinite gate gives an infinite gradient of the bias in its column: nothing behind the last row makes NaN of it."""
    rows, cols = 5, 40
    g = np.random.default_rng(4)
    y, d = (torch.from_numpy(np.abs(values(g, dtype, rows, cols)) + 0.5).to(TORCH[dtype]).cuda() for _ in range(2))
    gate = torch.ones(cols, dtype=TORCH[dtype], device="cuda")
    gate[7] = float("inf")
    got = back(y, None, d, None, dict(gate=gate), au.RMS, False, False, 0.0, None)
    assert got["dbias"][7] == float("inf") and got["dy"][:, 7].isinf().all()
    rest = [c for c in range(cols) if c != 7]
    assert all(got[v][..., rest].isfinite().all() for v in ("dbias", "dgate", "dy", "dx")) and got["dgate"].isfinite().all()
