"""The resized product with bias, activation, gate, dropout and residual, and its gradients, on the GPU, against the definition in
64 bits (bounds derived in act_util.py), in every layout and mode, at ragged sizes, pitches and alignments."""
import numpy as np
import pytest
import torch

import act_util as au

pytestmark = pytest.mark.gpu
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
SEED, OFFSET = 0x0123456789ABCDEF, 0xFEDCBA98765


def rng_of(seed=SEED, offset=OFFSET):
    wrap = lambda v: v - (1 << 64) if v >> 63 else v        # noqa: E731
    return torch.tensor([wrap(seed), wrap(offset)], dtype=torch.int64, device="cuda")


class Mat:
    """A matrix with a pitch of its own inside a buffer of canaries, off 16 bytes where asked."""

    def __init__(self, a, dtype, pad=0, off=0, fill=None):
        rows, cols = a.shape
        self.buf = torch.full(((rows + 2) * (cols + pad) + off + 8,), 12.5, dtype=TORCH[dtype], device="cuda")
        self.t = self.buf[off + cols + pad:off + cols + pad + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        self.t.copy_(torch.from_numpy(np.ascontiguousarray(a)).to(TORCH[dtype]))
        self.outside = torch.ones_like(self.buf, dtype=torch.bool)
        self.outside[off + cols + pad:off + cols + pad + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = False

    def check(self, name):
        assert (self.buf[self.outside] == 12.5).all(), f"{name}: written outside"

    def np(self):
        return self.t.double().cpu().numpy()


def values(g, dtype, *shape, size=1.0):
    return torch.from_numpy(g.standard_normal(shape) * size).to(TORCH[dtype]).double().numpy()


def within(got, want, bound, name):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got - want) / bound):.3g} bounds at {np.argwhere(bad)[:3].tolist()}"


def keep_of(g, n, ratio):
    k = max(1, int(np.floor((1 - ratio) * n + 0.5)))
    return np.sort(g.permutation(n)[:k])


def layer(M, K, N, dtype, mode_k, ratio, kn, act, bias, gate, p, residual, pad=0, off=0, workspace=True, seed=0, keep=None, split=False):
    """Forward and backward, checked."""
    from paper_2401_11469_amd import zr
    g = np.random.default_rng(seed + 1000 * M + K + N)
    X, W = values(g, dtype, M, K), values(g, dtype, K, N, size=1.5 / np.sqrt(K))
    b = values(g, dtype, N) if bias else None
    G = values(g, dtype, M, N) if gate else None
    R = values(g, dtype, M, N) if residual else None
    dY = values(g, dtype, M, N)
    if keep is None:
        keep = keep_of(g, K if mode_k else N, ratio)
    f = au.factor(SEED, OFFSET, M, N, p)
    mats = {n: Mat(a, dtype, pad, off) for n, a in (("X", X), ("W", W if kn else W.T), ("G", G), ("R", R), ("dY", dY)) if a is not None}
    get = lambda n: mats[n].t if n in mats else None        # noqa: E731
    dev = None if len(keep) == (K if mode_k else N) else torch.from_numpy(keep.astype(np.int32)).cuda()
    mode, layout = zr.DROP_K if mode_k else zr.DROP_N, zr.W_KN if kn else zr.W_NK
    bv = None if b is None else torch.from_numpy(b).to(TORCH[dtype]).cuda()
    outs = {n: Mat(np.zeros(s), dtype, pad, off) for n, s in (("Y", (M, N)), ("Z", (M, N)), ("dX", (M, K)), ("dW", (K, N) if kn else (N, K)), ("dG", (M, N)))}
    how = dict(mode=mode, act=act, gate=get("G"), p=p, rng=rng_of() if p else None, w_layout=layout)
    ws = None
    if workspace:
        ws = torch.empty(zr.act_workspace_bytes(M, K, N, len(keep), mode, TORCH[dtype]), dtype=torch.uint8, device="cuda")
    print(f"layer {M} x {K} x {N} {dtype} mode_k={mode_k} kept={len(keep)} kn={kn} act={act} p={p} pad={pad} off={off}", flush=True)
    zr.resized_linear_act_fwd(get("X"), get("W"), dev, bias=bv, residual=get("R"), Y=outs["Y"].t, Z=outs["Z"].t, workspace=ws, **how)
    torch.cuda.synchronize()
    (y, ey), (z, ez) = au.product(X, W, keep, mode_k, b, act, G, f, R, dtype)
    within(outs["Z"].np(), z, ez, "Z")
    within(outs["Y"].np(), y, ey, "Y")
    # without Z, and without scratch where there was some: the same bits, unless kept columns were extracted or the contraction split there
    Y2 = zr.resized_linear_act_fwd(get("X"), get("W"), dev, bias=bv, residual=get("R"), **how)
    if not (workspace and (split or mode_k and dev is not None)):
        assert torch.equal(Y2, outs["Y"].t)
    else:
        within(Y2.double().cpu().numpy(), y, ey, "Y without scratch")

    Z = outs["Z"].np()
    db = torch.zeros(N, dtype=TORCH[dtype], device="cuda") if bias else None
    zr.resized_linear_act_bwd(get("X"), get("W"), get("dY"), dev, Z=outs["Z"].t, dX=outs["dX"].t, dW=outs["dW"].t, dbias=db,
                              dgate=outs["dG"].t if gate else None, **how)
    torch.cuda.synchronize()
    dX, dW, dB, dG = au.product_back(X, W, dY, Z, keep, mode_k, act, G, f, dtype)
    within(outs["dX"].np(), *dX, "dX")
    within(outs["dW"].np() if kn else outs["dW"].np().T, *dW, "dW")
    if bias:
        within(db.double().cpu().numpy(), *dB, "dbias")
    if gate:
        within(outs["dG"].np(), *dG, "dgate")
    for n, m in list(mats.items()) + list(outs.items()):
        m.check(n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mode_k,kn", [(0, 0), (1, 1), (0, 1), (1, 0)])
@pytest.mark.parametrize("M,K,N,ratio", [(1, 1, 1, 0.0), (1, 64, 40, 0.25), (2, 7, 9, 0.3), (5, 264, 72, 0.5), (13, 100, 333, 0.1), (16, 512, 256, 0.0),
                                         (17, 129, 65, 0.25), (64, 96, 128, 0.0), (200, 328, 264, 0.25), (257, 130, 515, 0.4)])
def test_layer(M, K, N, ratio, mode_k, kn, dtype):
    layer(M, K, N, dtype, mode_k, ratio, kn, au.SILU, True, True, 0.1, True)


@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bias,gate,p,residual", [(0, 0, 0.0, 0), (1, 0, 0.0, 0), (0, 1, 0.0, 0), (0, 0, 0.5, 0), (0, 0, 0.0, 1), (1, 1, 0.9, 1)])
def test_each_part(act, dtype, bias, gate, p, residual):
    layer(33, 72, 88, dtype, False, 0.25, False, act, bias, gate, p, residual, seed=act)
    layer(3, 72, 88, dtype, True, 0.25, True, act, bias, gate, p, residual, seed=act)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mode_k,kn", [(0, 0), (1, 1), (0, 1), (1, 0)])
@pytest.mark.parametrize("pad,off", [(0, 1), (3, 0), (8, 0), (8, 8), (1, 3)])
def test_pitches_and_alignments(dtype, mode_k, kn, pad, off):
    layer(40, 136, 120, dtype, mode_k, 0.3, kn, au.GELU_TANH, True, True, 0.2, True, pad, off)
    layer(7, 136, 120, dtype, mode_k, 0.3, kn, au.GELU_TANH, True, True, 0.2, True, pad, off)


@pytest.mark.parametrize("mode_k,kn,M,K,N,ratio", [
    (0, 0, 512, 256, 1024, 0.25), (1, 1, 512, 1024, 512, 0.25), (0, 0, 1024, 192, 1280, 0.0), (1, 1, 1000, 320, 1032, 0.0),
    (0, 0, 2048, 128, 4096, 0.1), (1, 1, 2056, 256, 4104, 0.4), (0, 0, 2304, 328, 4000, 0.5), (0, 1, 768, 256, 768, 0.2), (1, 0, 768, 256, 768, 0.2)])
def test_many_tiles(mode_k, kn, M, K, N, ratio):
    layer(M, K, N, "bf16", mode_k, ratio, kn, au.GELU, True, True, 0.1, True)


@pytest.mark.parametrize("mode_k,kn,M,K,N,ratio", [(0, 0, 8192, 72, 2752, 0.25), (1, 1, 4096, 192, 4128, 0.25), (0, 1, 4096, 64, 4112, 0.0), (0, 0, 2112, 128, 8192, 0.0),
                                                   (0, 0, 4200, 128, 5120, 0.2), (1, 1, 6144, 136, 3000, 0.0)])
@pytest.mark.parametrize("workspace", [False, True])
def test_panels_of_whole_rounds_and_what_they_leave(mode_k, kn, M, K, N, ratio, workspace):
    layer(M, K, N, "bf16", mode_k, ratio, kn, au.SILU, True, True, 0.1, True, workspace=workspace)


@pytest.mark.parametrize("mode_k,kn,M,K,N,ratio", [(0, 0, 200, 4096, 256, 0.25), (1, 1, 384, 2752, 512, 0.25), (0, 0, 130, 1536, 1000, 0.0), (1, 1, 128, 5120, 128, 0.0)])
def test_split_contractions(mode_k, kn, M, K, N, ratio):
    layer(M, K, N, "bf16", mode_k, ratio, kn, au.GELU, True, True, 0.1, True, split=True)


@pytest.mark.parametrize("M", [1, 2, 4, 5, 8, 9, 16])
@pytest.mark.parametrize("mode_k,kn,K,N,ratio", [(0, 0, 4096, 2752, 0.0), (0, 0, 1000, 2000, 0.3), (1, 1, 2752, 4096, 0.0), (1, 1, 2752, 1024, 0.25), (1, 1, 1001, 520, 0.0),
                                                 (0, 0, 8, 4, 0.0), (0, 0, 7168, 40, 0.5), (1, 1, 7000, 8, 0.5)])
def test_few_rows(M, mode_k, kn, K, N, ratio):
    layer(M, K, N, "bf16", mode_k, ratio, kn, au.SILU, True, True, 0.1, True, workspace=M % 2 == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kept", ["first", "last", "one", "ends", "gap"])
def test_clustered_lists(dtype, kept):
    # long dropped ranges: their columns hold act(bias) * gate and so on
    for M, K, N in ((20, 64, 1500), (300, 64, 2600)):
        keep = {"first": np.arange(40), "last": np.arange(N - 40, N), "one": np.array([N // 2 + 3]), "ends": np.array([0, N - 1]),
                "gap": np.concatenate([np.arange(130), np.arange(N - 131, N)])}[kept]
        layer(M, K, N, dtype, False, 0, False, au.SILU, True, True, 0.1, True, keep=keep)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place(dtype):
    """Y may be the residual or the gate, dgate the gate, Z or dY."""
    from paper_2401_11469_amd import zr
    g = np.random.default_rng(5)
    for M, K, N, ratio in ((30, 64, 90, 0.3), (3, 64, 90, 0.0), (700, 64, 900, 0.3)):
        X, W, G, R, Z, dY = (torch.from_numpy(values(g, dtype, *s)).to(TORCH[dtype]).cuda() for s in ((M, K), (N, K), (M, N), (M, N), (M, N), (M, N)))
        keep = torch.from_numpy(keep_of(g, N, ratio).astype(np.int32)).cuda() if ratio else None
        how = dict(keep_idx=keep, mode=zr.DROP_N, act=au.SILU, p=0.2, rng=rng_of(), w_layout=zr.W_NK)
        want = zr.resized_linear_act_fwd(X, W, gate=G, residual=R, **how)
        Y = R.clone()
        assert torch.equal(zr.resized_linear_act_fwd(X, W, gate=G, residual=Y, Y=Y, **how), want)
        Y = G.clone()
        assert torch.equal(zr.resized_linear_act_fwd(X, W, gate=Y, residual=R, Y=Y, **how), want)
        dG = torch.empty_like(G)
        wx, ww = zr.resized_linear_act_bwd(X, W, dY, Z=Z, gate=G, dgate=dG, **how)
        for name in ("gate", "Z", "dY"):
            t = {"gate": G, "Z": Z, "dY": dY}[name].clone()
            args = {"gate": G, "Z": Z, "dY": dY, name: t}
            gx, gw = zr.resized_linear_act_bwd(X, W, args["dY"], Z=args["Z"], gate=args["gate"], dgate=t, **how)
            assert torch.equal(t, dG) and torch.equal(gx, wx) and torch.equal(gw, ww), name


def test_the_gate_gradient_of_a_plain_layer_over_dY():
    """No activation, gate or dropout: dZ is dY, which dgate may replace."""
    from paper_2401_11469_amd import zr
    g = np.random.default_rng(16)
    for dtype in ("bf16", "f32"):
        M, K, N = 40, 64, 96
        X, W, Z, dY = (torch.from_numpy(values(g, dtype, *s)).to(TORCH[dtype]).cuda() for s in ((M, K), (K, N), (M, N), (M, N)))
        wx, ww = zr.resized_linear_act_bwd(X, W, dY)
        want = torch.empty_like(dY)
        zr.resized_linear_act_bwd(X, W, dY, Z=Z, dgate=want)
        t = dY.clone()
        gx, gw = zr.resized_linear_act_bwd(X, W, t, Z=Z, dgate=t)
        assert torch.equal(gx, wx) and torch.equal(gw, ww) and torch.equal(t, want)
        within(t.double().cpu().numpy(), (dY.double() * Z.double()).cpu().numpy(), au.U[dtype] * (dY.double() * Z.double()).abs().cpu().numpy() * 1.01, "dgate")


def test_which_outputs_are_wanted_changes_none():
    from paper_2401_11469_amd import zr
    g = np.random.default_rng(6)
    M, K, N = 50, 72, 104
    X, W, G, Z, dY = (torch.from_numpy(values(g, "bf16", *s)).bfloat16().cuda() for s in ((M, K), (K, N), (M, N), (M, N), (M, N)))
    keep = torch.from_numpy(keep_of(g, K, 0.25).astype(np.int32)).cuda()
    how = dict(keep_idx=keep, mode=zr.DROP_K, act=au.GELU, Z=Z, gate=G, p=0.1, rng=rng_of())
    db, dG = torch.empty(N, dtype=torch.bfloat16, device="cuda"), torch.empty_like(Z)
    dX, dW = zr.resized_linear_act_bwd(X, W, dY, dbias=db, dgate=dG, **how)
    assert torch.equal(zr.resized_linear_act_bwd(X, W, dY, need_dW=False, **how)[0], dX)
    assert torch.equal(zr.resized_linear_act_bwd(X, W, dY, need_dX=False, **how)[1], dW)
    db2, dG2 = torch.empty_like(db), torch.empty_like(dG)
    assert zr.resized_linear_act_bwd(None, W, dY, need_dX=False, need_dW=False, dbias=db2, **how) == (None, None)
    zr.resized_linear_act_bwd(None, W, dY, need_dX=False, need_dW=False, dgate=dG2, **how)
    assert torch.equal(db, db2) and torch.equal(dG, dG2)
    # no activation, gate or dropout: the gradients of the plain layer, and the sums of dY
    a, b = zr.resized_linear_act_bwd(X, W, dY, keep, zr.DROP_K, dbias=db)
    ws = torch.empty(zr.workspace_bytes(M, K, N, keep.numel(), zr.DROP_K, torch.bfloat16), dtype=torch.uint8, device="cuda")
    wx, ww = zr.resized_linear_bwd(X, W, dY, keep, zr.DROP_K, workspace=ws)
    assert torch.equal(a, wx) and torch.equal(b, ww)
    want = dY.double().sum(0)
    assert ((db.double() - want).abs() <= 2.0 ** -8 * want.abs() + 8 * 50 ** 0.5 * au.F * dY.double().norm(dim=0)).all()


def test_masked_places_hold_anything():
    """A dropped element is the residual alone, whatever gate and sum are there; NaN and infinity elsewhere go their way."""
    from paper_2401_11469_amd import zr
    g = np.random.default_rng(7)
    M, K, N, p = 24, 40, 72, 0.5
    f = au.factor(SEED, OFFSET, M, N, p)
    for dtype in ("bf16", "f32"):
        X, W, G, R = (torch.from_numpy(values(g, dtype, *s)).to(TORCH[dtype]).cuda() for s in ((M, K), (K, N), (M, N), (M, N)))
        mask = torch.from_numpy(f == 0).cuda()
        want = zr.resized_linear_act_fwd(X, W, act=au.SILU, gate=G, residual=R, p=p, rng=rng_of())
        for bad in (float("nan"), float("inf"), -float("inf")):
            Gb = torch.where(mask, torch.full_like(G, bad), G)
            assert torch.equal(zr.resized_linear_act_fwd(X, W, act=au.SILU, gate=Gb, residual=R, p=p, rng=rng_of()), want)
            y = zr.resized_linear_act_fwd(X, W, act=au.RELU, gate=torch.where(mask, G, torch.full_like(G, bad)), p=p, rng=rng_of())
            assert (y[mask] == 0).all()
            dYb = torch.where(mask, torch.full_like(G, bad), G)
            dX, dW = zr.resized_linear_act_bwd(X, W, dYb, act=au.SILU, Z=R, p=p, rng=rng_of())
            assert dX.isfinite().all() and dW.isfinite().all()


@pytest.mark.parametrize("act", range(1, 5))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_activation_at_its_ends(act, dtype):
    """Large arguments of either sign, zeros, NaN: through an identity product."""
    from paper_2401_11469_amd import zr
    z = np.array([0.0, -0.0, 1e-30, -1e-30, 1e-3, -1e-3, 5, -5, 12, -12, 30, -30, 88, -88, 200, -200, 1e4, -1e4, 3e38, -3e38, 0.75, -0.75, 2, -2])
    t = torch.from_numpy(z).to(TORCH[dtype])
    z = t.double().numpy()[None]
    X = torch.ones(1, 1, dtype=TORCH[dtype], device="cuda")
    Y = zr.resized_linear_act_fwd(X, t.cuda()[None].contiguous(), act=act)
    with np.errstate(over="ignore", under="ignore", invalid="ignore"):
        a, s = au.act(act, z)
        ok = np.abs(z) < 1e4 if act == au.GELU_TANH else np.abs(z) < 1e18         # (z^3, z^2 in 32 bits)
        ea, es = au.act_error(act, z, a)
        got = Y.double().cpu().numpy()
        within(np.where(ok, got, 0), np.where(ok, a, 0), ea + 2.0 ** -8 * abs(a) + 1e-37, "value")
        dW = zr.resized_linear_act_bwd(X, t.cuda()[None].contiguous(), torch.ones_like(Y), act=act, Z=t.cuda()[None].contiguous(), need_dX=False)[1]
        ok &= np.abs(z) < 1e3
        within(np.where(ok, dW.double().cpu().numpy(), 0), np.where(ok, s, 0), np.where(np.abs(z) > 30, 1e-30, es) + 2 * 2.0 ** -8 * abs(s) + 1e-37, "slope")
    up = torch.full((1, 8), float("inf"), dtype=TORCH[dtype], device="cuda")
    assert torch.equal(zr.resized_linear_act_fwd(X, up, act=act), up)
    nan = torch.full((1, 8), float("nan"), dtype=TORCH[dtype], device="cuda")
    assert zr.resized_linear_act_fwd(X, nan, act=act).isnan().all()


@pytest.mark.parametrize("act", range(1, 5))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_slope_of_large_values(act, dtype):
    """The slope is 1 or 0 there, also where z^2 is past the largest fp32 number."""
    from paper_2401_11469_amd import zr
    big = torch.tensor([1e6, 1e19, 1e20, 1e30, 3e38], dtype=TORCH[dtype], device="cuda")
    z = torch.cat([big, -big])[None]
    dY, out = torch.ones_like(z), torch.empty_like(z)
    W = torch.eye(10, dtype=TORCH[dtype], device="cuda")
    dX, _ = zr.resized_linear_act_bwd(None, W, dY, mode=zr.DROP_N, act=act, Z=z, dgate=out, need_dW=False)
    assert dX.cpu().tolist() == [[1.0] * 5 + [0.0] * 5]
    assert torch.equal(out, z.clamp(min=0))


def test_another_stream_and_repeatability():
    from paper_2401_11469_amd import zr
    g = np.random.default_rng(8)
    M, K, N = 500, 264, 520
    X, W, dY = (torch.from_numpy(values(g, "bf16", *s)).bfloat16().cuda() for s in ((M, K), (N, K), (M, N)))
    keep = torch.from_numpy(keep_of(g, N, 0.25).astype(np.int32)).cuda()
    how = dict(keep_idx=keep, mode=zr.DROP_N, act=au.GELU, p=0.1, rng=rng_of(), w_layout=zr.W_NK)

    def both(stream=None):
        Z = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
        db = torch.empty(N, dtype=torch.bfloat16, device="cuda")
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        Y = zr.resized_linear_act_fwd(X, W, Z=Z, stream=stream, **how)
        dX, dW = zr.resized_linear_act_bwd(X, W, dY, Z=Z, dbias=db, stream=stream, **how)
        if stream is not None:
            torch.cuda.current_stream().wait_stream(stream)
        return Y, Z, dX, dW, db

    want = both()
    for s in (None, torch.cuda.Stream(), torch.cuda.Stream()):
        for a, b in zip(both(s), want):
            assert torch.equal(a, b)


def test_binding_refusals():
    from paper_2401_11469_amd import zr
    b = torch.bfloat16
    X, W, G = torch.zeros(4, 16, dtype=b, device="cuda"), torch.zeros(16, 8, dtype=b, device="cuda"), torch.zeros(4, 8, dtype=b, device="cuda")
    bad = [dict(W=W.float()), dict(W=W.t()), dict(X=X.cpu()), dict(X=X[:, ::2]), dict(bias=torch.zeros(7, dtype=b, device="cuda")),
           dict(bias=torch.zeros(8, device="cuda")), dict(bias=torch.zeros(16, dtype=b, device="cuda")[::2]), dict(gate=X), dict(gate=G.float()),
           dict(residual=G.cpu()), dict(Y=X), dict(Z=G.t()), dict(p=0.1, rng=torch.zeros(2, device="cuda")),
           dict(p=0.1, rng=torch.zeros(2, dtype=torch.int64)), dict(p=0.1, rng=torch.zeros(3, dtype=torch.int64, device="cuda")), dict(p=0.1), dict(p=1.0),
           dict(act=9), dict(keep_idx=torch.zeros(4, dtype=torch.int64, device="cuda")), dict(keep_idx=torch.zeros(0, dtype=torch.int32, device="cuda")),
           dict(workspace=torch.zeros(64, dtype=torch.uint8))]
    zr.resized_linear_act_fwd(X, W)
    for change in bad:
        with pytest.raises((ValueError, RuntimeError, TypeError)):
            zr.resized_linear_act_fwd(**{**dict(X=X, W=W), **change})
    for change in (dict(dY=X), dict(Z=None), dict(X=None), dict(dX=G), dict(dW=G), dict(dbias=torch.zeros(9, dtype=b, device="cuda")), dict(dgate=X),
                   dict(workspace=torch.zeros(48, dtype=torch.uint8, device="cuda"))):      # (dZ: 64 bytes)
        with pytest.raises((ValueError, RuntimeError, TypeError)):
            zr.resized_linear_act_bwd(**{**dict(X=X, W=W, dY=G, Z=G, act=zr.ACT_SILU), **change})
