"""Dropout, and a block's output joining the residual stream with its norms, forward and backward, on the GPU, against the
definitions in 64 bits (bounds derived in act_util.py)."""
import numpy as np
import pytest
import torch

import act_util as au
from test_gpu_act import OFFSET, SEED, TORCH, Mat, rng_of, values, within

pytestmark = pytest.mark.gpu


# ---- dropout ----
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pad,off", [(1, 1, 0, 0), (1, 8, 0, 0), (3, 7, 0, 1), (197, 1023, 0, 0), (5, 64, 3, 2), (33, 513, 1, 0), (1000, 40, 0, 0),
                                               (2, 9000, 8, 0), (4097, 24, 0, 0)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.99999])
def test_dropout(dtype, rows, cols, pad, off, p):
    from paper_2401_11469_amd import zr
    g = np.random.default_rng(rows + cols)
    x = values(g, dtype, rows, cols)
    X, out = Mat(x, dtype, pad, off), Mat(np.zeros_like(x), dtype, pad, off)
    zr.dropout(X.t, p, rng_of(), out=out.t)
    f = au.factor(SEED, OFFSET, rows, cols, p)
    want = au.times(f, x)
    within(out.np(), want, np.abs(want) * (au.F + au.U[dtype]) * 1.01, "out")
    assert (out.np()[f == 0] == 0).all() and not torch.signbit(out.t.cpu()[torch.from_numpy(f == 0)]).any()
    out.check("out")
    # in place, and dropped places hold anything
    Y = X.t.clone()
    Y[torch.from_numpy(f == 0).cuda()] = float("nan")
    assert torch.equal(zr.dropout(Y, p, rng_of(), out=Y), out.t)


def test_dropout_draws_by_seed_offset_row_and_column():
    from paper_2401_11469_amd import zr
    x = torch.ones(64, 96, device="cuda")
    a = zr.dropout(x, 0.5, rng_of())
    assert torch.equal(a, zr.dropout(x, 0.5, rng_of()))
    seen = [a]
    for seed, offset in ((SEED + 1, OFFSET), (SEED, OFFSET + 1), (SEED ^ (1 << 63), OFFSET), (SEED, OFFSET ^ (1 << 40))):
        b = zr.dropout(x, 0.5, rng_of(seed, offset))
        for c in seen:
            assert 0.4 < (b == c).float().mean() < 0.6          # 6144 coins: 0.5 by 15 standard deviations
        seen.append(b)
    # a part of the columns and rows draws what the whole does
    assert torch.equal(zr.dropout(x[:10, :40], 0.5, rng_of()), a[:10, :40])


def test_dropout_past_32_bits_of_elements():
    from paper_2401_11469_amd import zr
    rows, cols = 524304, 4104
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    zr.dropout(x, 0.25, rng_of(), out=x)
    for r in (0, 300000, 523270, rows - 4):
        f = np.where(au.halves(SEED, OFFSET, 4, cols, first_row=r) >= 16384, 4 / 3, 0.0)
        within(x[r:r + 4].double().cpu().numpy(), f, f * 2.0 ** -8, r)
    del x


def test_dropout_refusals():
    from paper_2401_11469_amd import zr
    x = torch.zeros(4, 8, device="cuda")
    for args in ((x, 0.1, None), (x, 1.0, rng_of()), (x, -1.0, rng_of()), (x.cpu(), 0.1, rng_of()), (x.t(), 0.1, rng_of()), (x[0], 0.1, rng_of()),
                 (x.half(), 0.1, rng_of()), (x, 0.1, rng_of().cpu()), (x, 0.1, rng_of().int())):
        with pytest.raises((ValueError, RuntimeError, TypeError)):
            zr.dropout(*args)
    with pytest.raises(ValueError):
        zr.dropout(x, 0.1, rng_of(), out=x.bfloat16())


# ---- joins ----
VECTORS = ("bias", "gate", "post_w", "post_b", "pre_w", "pre_b")


def join(rows, cols, dtype, kind, post, pre, p=0.0, scale=1.0, vectors=VECTORS, pad=0, off=0, eps=1e-5, dxo=True, mean=0.0, seed=0):
    from paper_2401_11469_amd import zr
    g = np.random.default_rng(seed + rows * 7 + cols)
    y, x = values(g, dtype, rows, cols) , values(g, dtype, rows, cols, size=2.0)
    x = torch.from_numpy(x + mean).to(TORCH[dtype]).double().numpy()
    vec = {v: values(g, dtype, cols) for v in vectors if v in ("bias", "gate") or (post if v.startswith("post") else pre)}
    dev = {v: torch.from_numpy(a).to(TORCH[dtype]).cuda() for v, a in vec.items()}
    f = au.factor(SEED, OFFSET, rows, cols, p)
    Y, X, XO, H = (Mat(a, dtype, pad, off) for a in (y, x, 0 * x, 0 * x))
    how = dict(norm=kind, post=post, pre=pre, eps=eps, p=p, rng=rng_of() if p else None, scale=scale)
    print(f"join {rows} x {cols} {dtype} kind={kind} post={post} pre={pre} p={p} vectors={sorted(vec)} pad={pad} off={off}", flush=True)
    zr.block_join_fwd(Y.t, X.t, **how, **dev, x_out=XO.t, h=H.t if pre else None)
    torch.cuda.synchronize()
    want = au.join(y, x, kind, post, pre, eps, f, scale, vec, dtype)
    within(XO.np(), *want[0], "x_out")
    if pre:
        within(H.np(), *want[1], "h")

    d, dh = values(g, dtype, rows, cols), values(g, dtype, rows, cols)
    D, DH, DX, DY = (Mat(a, dtype, pad, off) for a in (d, dh, 0 * x, 0 * x))
    dxo = dxo or not pre
    grads = {v: torch.empty(cols, dtype=TORCH[dtype], device="cuda") for v in vec}
    zr.block_join_bwd(D.t if dxo else None, DH.t if pre else None, XO.t if pre else None, Y.t, **how, **{v: t for v, t in dev.items() if v != "pre_b"},
                      dx=DX.t, dy=DY.t, **{"d" + v: t for v, t in grads.items()})
    torch.cuda.synchronize()
    back = au.unjoin(d if dxo else None, dh, XO.np(), y, kind, post, pre, eps, f, scale, vec, dtype)
    within(DX.np(), *back["dx"], "dx")
    within(DY.np(), *back["dy"], "dy")
    for v, t in grads.items():
        within(t.double().cpu().numpy(), *back[v], "d" + v)
    for m in (Y, X, XO, H, D, DH, DX, DY):
        m.check("join")


BOTH = [(False, False), (True, False), (False, True), (True, True)]


@pytest.mark.parametrize("post,pre", BOTH)
@pytest.mark.parametrize("kind", [au.RMS, au.LAYER])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 5), (2, 8), (3, 63), (5, 512), (9, 513), (197, 1000), (6, 1024), (7, 1025), (40, 2048), (3, 2049),
                                       (33, 4096), (2, 4100), (5, 8192), (4, 8200), (3, 16384)])
def test_join(rows, cols, dtype, kind, post, pre):
    join(rows, cols, dtype, kind, post, pre, p=0.1, scale=0.7)


@pytest.mark.parametrize("post,pre", BOTH)
@pytest.mark.parametrize("vectors", [(), ("bias",), ("gate",), ("post_w", "pre_w"), ("post_b", "pre_b"), ("bias", "post_w", "pre_b")])
def test_vectors_that_are_missing(post, pre, vectors):
    for dtype in ("bf16", "f32"):
        join(21, 130, dtype, au.LAYER, post, pre, vectors=vectors)
        join(21, 1300, dtype, au.RMS, post, pre, p=0.3, vectors=vectors, dxo=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad,off", [(1, 0), (0, 1), (8, 8), (3, 5)])
def test_pitches(dtype, pad, off):
    for cols in (64, 777, 1536, 3000):
        join(11, cols, dtype, au.LAYER, True, True, p=0.2, scale=-1.5, pad=pad, off=off)


@pytest.mark.parametrize("rows,cols", [(3000, 100), (5000, 768), (2500, 1400), (1200, 4000), (700, 5000)])
def test_more_rows_than_places(rows, cols):
    join(rows, cols, "bf16", au.RMS, True, True, p=0.1)
    join(rows, cols, "f32", au.LAYER, False, True)


def test_a_large_mean_and_equal_values():
    join(9, 700, "f32", au.LAYER, False, True, mean=100.0)
    join(9, 700, "bf16", au.LAYER, True, True, mean=30.0)
    from paper_2401_11469_amd import zr
    # a row of equal values has no deviation: layer norm gives the bias, of either sign of zero or not
    x = torch.full((3, 96), 2.5, device="cuda")
    b = torch.linspace(-1, 1, 96, device="cuda")
    xo, h = zr.block_join_fwd(torch.zeros_like(x), x, norm=zr.NORM_LAYER, pre_b=b)
    assert torch.equal(xo, x) and torch.equal(h, b.expand(3, 96))
    # a row of zeros under a root mean square: zeros, and gradients of 1 / sqrt(eps)
    z = torch.zeros_like(x)
    xo, h = zr.block_join_fwd(z, z, norm=zr.NORM_RMS, eps=1e-4)
    assert (h == 0).all()
    dx, dy = zr.block_join_bwd(None, torch.ones_like(x), xo, None, norm=zr.NORM_RMS, eps=1e-4)
    assert ((dx - 100).abs() <= 100 * 2.0 ** -21).all() and torch.equal(dx, dy)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [200, 1500, 6000])
def test_in_place(dtype, cols):
    from paper_2401_11469_amd import zr
    g = np.random.default_rng(cols)
    y, x, d, dh = (torch.from_numpy(values(g, dtype, 13, cols)).to(TORCH[dtype]).cuda() for _ in range(4))
    how = dict(norm=zr.NORM_LAYER, post=True, pre=True, p=0.1, rng=rng_of(), scale=0.5)
    xo, h = zr.block_join_fwd(y, x, **how)
    a = x.clone()
    b = y.clone()
    got = zr.block_join_fwd(b, a, x_out=a, h=b, **how)
    assert torch.equal(got[0], xo) and torch.equal(got[1], h)
    b = y.clone()
    got = zr.block_join_fwd(b, x, x_out=b, **how)
    assert torch.equal(got[0], xo) and torch.equal(got[1], h)
    dx, dy = zr.block_join_bwd(d, dh, xo, y, **how)
    for name in ("d", "dh", "xo"):
        args = dict(d=d.clone(), dh=dh.clone(), xo=xo.clone())
        b = y.clone()
        got = zr.block_join_bwd(args["d"], args["dh"], args["xo"], b, dx=args[name], dy=b, **how)
        assert torch.equal(got[0], dx) and torch.equal(got[1], dy), name


def test_which_outputs_are_wanted_changes_none():
    from paper_2401_11469_amd import zr
    g = np.random.default_rng(9)
    rows, cols = 300, 1100
    y, xo, d, dh = (torch.from_numpy(values(g, "bf16", rows, cols)).bfloat16().cuda() for _ in range(4))
    w = {v: torch.from_numpy(values(g, "bf16", cols)).bfloat16().cuda() for v in ("bias", "gate", "post_w", "post_b", "pre_w")}
    how = dict(norm=zr.NORM_RMS, post=True, pre=True, p=0.1, rng=rng_of(), **w)
    all_ = {"d" + v: torch.empty(cols, dtype=torch.bfloat16, device="cuda") for v in VECTORS}
    dx, dy = zr.block_join_bwd(d, dh, xo, y, **how, **all_)
    for v in all_:
        one = torch.empty_like(all_[v])
        assert zr.block_join_bwd(d, dh, xo, y, need_dx=False, need_dy=False, **how, **{v: one}) == (None, None)
        assert torch.equal(one, all_[v])
    assert torch.equal(zr.block_join_bwd(d, dh, xo, y, need_dy=False, **how)[0], dx)
    assert torch.equal(zr.block_join_bwd(d, dh, xo, y, need_dx=False, **how)[1], dy)


def test_join_past_32_bits_of_elements():
    from paper_2401_11469_amd import zr
    rows, cols = 530000, 4104
    y = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x = torch.ones_like(y)
    y[-3:] = 1.0
    xo, h = zr.block_join_fwd(y, x, scale=2.0, x_out=x, h=y, eps=0.0)
    assert (xo[-3:] == 3).all() and (xo[:-3:1000] == 1).all() and (h[::1000] == 1).all() and (h[-3:] == 1).all()
    del y, x, xo, h


def test_join_refusals():
    from paper_2401_11469_amd import zr
    x, v = torch.zeros(4, 8, device="cuda"), torch.zeros(8, device="cuda")
    zr.block_join_fwd(x, x.clone())
    for change in (dict(x=x.cpu()), dict(x=x.bfloat16()), dict(x=torch.zeros(4, 9, device="cuda")), dict(y=x.t()), dict(bias=v[:7]), dict(bias=v.bfloat16()),
                   dict(pre_w=torch.zeros(16, device="cuda")[::2]), dict(p=0.5), dict(p=0.5, rng=rng_of().cpu()), dict(norm=3), dict(eps=-1.0), dict(h=x[:3])):
        with pytest.raises((ValueError, RuntimeError, TypeError)):
            zr.block_join_fwd(**{**dict(y=x, x=x.clone()), **change})
    for change in (dict(dh=None), dict(x_out=None), dict(dx_out=None, dh=None), dict(dpost_w=v), dict(dgate=v, y=None), dict(dgate=v[:5]), dict(dx=x[:2]),
                   dict(dpre_w=v, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ValueError, RuntimeError, TypeError)):
            zr.block_join_bwd(**{**dict(dx_out=x, dh=x, x_out=x, y=x), **change})
    wide = torch.zeros(1, 16385, device="cuda")
    with pytest.raises(RuntimeError):
        zr.block_join_fwd(wide, wide.clone())
