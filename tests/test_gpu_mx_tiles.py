"""The block-scaled product on every kind of tile that its sizes choose (256 x 256 alone and with a panel of smaller ones,
128 x 128 with two and with four units in LDS, 64 x 64), with contractions of odd and even numbers of steps and of more than four
groups of scales; pitches whose offsets pass 32 bits; calls on two streams at once.  Against float64 products on the GPU, within the bounds of
test_gpu_mx.py."""
import numpy as np
import pytest

from mx_util import E2M1, E4M3
from parity_util import acc_term
from test_gpu_mx import DROP_K, DROP_N, SAME, U, ZERO, idx, subset
from test_gpu_mx import torch, zr  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu
PAIRS = [(E2M1, E2M1), (E4M3, E2M1), (E4M3, E4M3)]


def normal(torch, seed, *shape, dtype=None, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(shape, generator=g, device="cuda") * torch.exp(0.4 * torch.randn(shape[-1:], generator=g, device="cuda")) * scale
    return x.to(dtype or torch.bfloat16)


def check(torch, got, xv, wv, dtype, cut, rows=2048):
    """got [M, J] against xv [M, C] wv [J, C]^T (float64 on the GPU), a part of the rows at a time."""
    C = xv.shape[1]
    pad = -C % 8
    top = lambda v: torch.nn.functional.pad(v.abs(), (0, pad)).view(v.shape[0], -1, 8).amax(dim=2)  # noqa: E731
    err = norm = 0.0
    for r in range(0, xv.shape[0], rows):
        x, g = xv[r:r + rows], got[r:r + rows].double()
        want = x @ wv.t()
        bound = (C + 8) * 2.0 ** -23 * (x.abs() @ wv.abs().t())
        if cut:
            bound += 8 * 2.0 ** -13 * (top(x) @ top(wv).t())
        bound = bound * (1 + U[dtype]) + U[dtype] * want.abs()
        off = (g - want).abs()
        assert torch.isfinite(g).all() and bool((off <= bound).all()), (r, float((off - bound).max()))
        err += float((g - want).square().sum())
        norm += float(want.square().sum())
    rel = (err / norm) ** 0.5
    assert rel <= (5e-3 if dtype == "bf16" else acc_term(C)), rel


@pytest.mark.parametrize("xf,wf", PAIRS)
@pytest.mark.parametrize("M,N,C", [(8192, 2048, 1000), (8190, 2041, 1100), (8192, 2048, 4500),      # 256 x 256
                                   (8192, 2064, 4100), (2100, 8192, 4100),                          # and a panel of the rest
                                   (4130, 4200, 700), (2200, 8300, 2500),                           # 128 x 128, two units
                                   (1500, 2100, 1024), (2048, 2000, 5000),                          # four units
                                   (600, 500, 3000), (100, 200, 5200), (17, 40, 2049)])             # 64 x 64
def test_every_kind_of_tile(torch, zr, M, N, C, xf, wf):  # noqa: F811
    X, W = normal(torch, M, M, C), normal(torch, N, N, C, scale=0.05)
    xm, wm = zr.mx_quantize(X, xf), zr.mx_quantize(W, wf)
    xv, wv = (zr.mx_dequantize(m, torch.float32).double() for m in (xm, wm))
    cut = xf == E4M3
    buf = torch.full((M + 1, N + 8), 77.0, dtype=torch.bfloat16, device="cuda")
    Y = buf[:M, :N]
    zr.mx_linear_fwd(xm, wm, Y=Y)
    check(torch, Y, xv, wv, "bf16", cut)
    assert torch.all(buf[M] == 77.0) and torch.all(buf[:M, N:] == 77.0)
    again = zr.mx_linear_fwd(xm, wm)
    assert torch.equal(again, Y)
    # three quarters of the features, the others as they were
    s = subset(N, N, N * 3 // 4)
    keep = idx(torch, s)
    prev = normal(torch, 5, M, N)
    Z = zr.mx_linear_fwd(xm, wm, keep, DROP_N, SAME, prev_Y=prev)
    check(torch, Z[:, keep.long()], xv, wv[keep.long()], "bf16", cut)
    drop = torch.ones(N, dtype=torch.bool, device="cuda")
    drop[keep.long()] = False
    assert torch.equal(Z[:, drop], prev[:, drop])
    Z = zr.mx_linear_fwd(xm, wm, keep, DROP_N, ZERO, Y=Y)
    assert torch.all(Z[:, drop] == 0) and torch.all(buf[M] == 77.0) and torch.all(buf[:M, N:] == 77.0)


@pytest.mark.parametrize("M,N,C", [(8192, 2064, 1500), (2048, 2000, 700), (900, 1100, 2300)])
@pytest.mark.parametrize("xf,wf", PAIRS)
def test_fp32_results(torch, zr, M, N, C, xf, wf):  # noqa: F811
    X, W = normal(torch, M, M, C, dtype=torch.float32), normal(torch, N, N, C, dtype=torch.float32, scale=0.05)
    wm = zr.mx_quantize(W, wf)
    ck = zr.mx_empty(M, C, xf)
    Y = zr.mx_linear_fwd(X, wm, x_fmt=xf, x_mx=ck)
    check(torch, Y, *(zr.mx_dequantize(m, torch.float32).double() for m in (ck, wm)), "f32", False)


def test_few_columns_of_many(torch, zr):  # noqa: F811
    """Tiles that own far more original columns than they have."""
    M, N, C = 700, 9000, 260
    X, W = normal(torch, 1, M, C), normal(torch, 2, N, C)
    xm, wm = zr.mx_quantize(X, E4M3), zr.mx_quantize(W, E2M1)
    xv, wv = (zr.mx_dequantize(m, torch.float32).double() for m in (xm, wm))
    for s in (np.array([4321], np.int32), np.r_[0:100, 8990:9000].astype(np.int32), subset(3, N, 130)):
        keep = idx(torch, s)
        for rows in (M, 9):
            x = zr.MX(xm.q[:rows], xm.scales[:rows], C, E4M3)
            Z = zr.mx_linear_fwd(x, wm, keep, DROP_N)
            check(torch, Z[:, keep.long()], xv[:rows], wv[keep.long()], "bf16", True)
            assert int((Z != 0).any(dim=0).sum()) <= s.size


def spread(torch, zr, m, pitch):  # noqa: F811
    """The same matrix with its rows `pitch` bytes apart."""
    rows = m.q.shape[0]
    q = torch.empty((rows, pitch), dtype=torch.uint8, device="cuda")
    q[:, :m.q.shape[1]] = m.q
    return zr.MX(q, m.scales, m.n, m.fmt)


@pytest.mark.parametrize("M,N,pitch", [(5000, 2100, 1 << 20), (300, 2100, 1 << 24)])
def test_offsets_beyond_32_bits(torch, zr, M, N, pitch):  # noqa: F811
    C = 2000
    X, W = normal(torch, 1, M, C), normal(torch, 2, N, C, scale=0.05)
    xm, wm = zr.mx_quantize(X, E4M3), zr.mx_quantize(W, E2M1)
    xv, wv = (zr.mx_dequantize(m, torch.float32).double() for m in (xm, wm))
    far = spread(torch, zr, xm, pitch)
    assert far.q.numel() > 2 ** 32
    check(torch, zr.mx_linear_fwd(far, wm), xv, wv, "bf16", True)
    assert torch.equal(zr.mx_dequantize(far), zr.mx_dequantize(xm))
    out = zr.MX(torch.zeros_like(far.q), xm.scales.clone(), C, E4M3)
    zr.mx_quantize(X, E4M3, out=out)
    assert torch.equal(out.q[:, :xm.q.shape[1]], xm.q) and torch.equal(out.scales, xm.scales)
    del far, out
    # rows of the weight picked from all over such a matrix
    s = subset(4, N, 1700)
    wfar = spread(torch, zr, wm, 1 << 21)
    assert wfar.q.numel() > 2 ** 32
    Z = zr.mx_linear_fwd(xm, wfar, idx(torch, s), DROP_N)
    k = torch.from_numpy(s).long().cuda()
    check(torch, Z[:, k], xv, wv[k], "bf16", True)


def test_two_streams_at_once(torch, zr):  # noqa: F811
    """Independent steps on two streams, nothing shared but the inputs."""
    M, K, N = 1000, 900, 1100
    X, W, dY = normal(torch, 1, M, K), normal(torch, 2, K, N, scale=0.05), normal(torch, 3, M, N)
    keep = idx(torch, subset(1, K, 700))

    def step(stream):
        wm = zr.mx_quantize(W, E2M1, axis=0, keep_idx=keep, out=zr.mx_empty(N, 700, E2M1), stream=stream)
        ck = zr.mx_empty(M, 700, E4M3)
        Y = zr.mx_linear_fwd(X, wm, keep, DROP_K, x_mx=ck, stream=stream)
        return (Y, *zr.resized_linear_bwd_mx(ck, W, dY, keep, DROP_K, stream=stream), wm, ck)

    want = step(None)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(6):
        for s in streams:
            got.append(step(s))
    torch.cuda.synchronize()
    for g in got:
        for a, b in zip(g[:3], want[:3]):
            assert torch.equal(a, b)


def test_captured_product_of_two_panels(torch, zr):  # noqa: F811
    """A product of two launches and one of the mean as the imputed value, replayed with other inputs."""
    M, N, C = 8192, 2064, 1400
    X, W = normal(torch, 1, M, C), normal(torch, 2, N, C, scale=0.05)
    wm = zr.mx_quantize(W, E4M3)
    keep = idx(torch, subset(1, N, 1500))
    ck, ek = zr.mx_empty(M, C, E4M3), zr.mx_empty(M, C, E4M3)
    outs = [torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(4)]

    def run(c, a, b):
        zr.mx_linear_fwd(X, wm, Y=a, x_mx=c)
        zr.mx_linear_fwd(c, wm, keep, DROP_N, 1, Y=b)

    run(ck, *outs[:2])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(ck, *outs[:2])
    for seed in range(3):
        X.copy_(normal(torch, 10 + seed, M, C))
        outs[0].fill_(3.0)
        outs[1].fill_(3.0)
        g.replay()
        run(ek, *outs[2:])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])
