"""Up to 16 rows of X: contractions that pass through LDS in more than one part (64 K of X in 8 bits, 128 K in 4, are one), with 8 and with
16 wavefronts to a workgroup, and more columns than the chip takes at once (256 workgroups of 16).  Against float64, within the bounds of test_gpu_mx.py; an input
that arrives in its own type and one in blocks give the same to the bit."""
import pytest

from mx_util import E2M1, E4M3
from test_gpu_mx import DROP_K, DROP_N, SAME, idx, subset, tdt
from test_gpu_mx import torch, zr  # noqa: F401  (fixtures)
from test_gpu_mx_tiles import check, normal

pytestmark = pytest.mark.gpu
PAIRS = [(E4M3, E2M1), (E2M1, E2M1), (E4M3, E4M3)]
# M, C: one value more than one part, a last part of a step, two and three parts, for 16, 9 and 1 rows
DEEP = [(16, 4097), (16, 5000), (16, 8192), (16, 11008), (16, 17000), (9, 7169), (9, 15000), (9, 30000), (1, 65537), (1, 140000)]


@pytest.mark.parametrize("xf,wf", PAIRS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,C", DEEP)
def test_contractions_of_several_parts(torch, zr, M, C, dtype, xf, wf):  # noqa: F811
    dt = tdt(torch, dtype)
    N = 100
    X, W = normal(torch, M + C, M, C, dtype=dt), normal(torch, C, N, C, dtype=dt, scale=0.05)
    wm, xm = zr.mx_quantize(W, wf), zr.mx_quantize(X, xf)
    xv, wv = (zr.mx_dequantize(m, torch.float32).double() for m in (xm, wm))
    Y = zr.mx_linear_fwd(X, wm, x_fmt=xf)
    check(torch, Y, xv, wv, dtype, dtype == "bf16" and xf == E4M3)
    assert torch.equal(zr.mx_linear_fwd(xm, wm, dtype=dt), Y)
    ck = zr.mx_empty(M, C, xf)
    assert torch.equal(zr.mx_linear_fwd(X, wm, x_fmt=xf, x_mx=ck), Y) and torch.equal(ck.q, xm.q) and torch.equal(ck.scales, xm.scales)
    # rows that no vector load fits, and a kept part of the contraction
    off = torch.empty(M * (C + 1) + 1, dtype=dt, device="cuda")[1:].view(M, C + 1)[:, :C]
    off.copy_(X)
    assert torch.equal(zr.mx_linear_fwd(off, wm, x_fmt=xf), Y)
    n = C - 5
    keep = idx(torch, subset(C, C, n))
    wk, xk = zr.mx_quantize(W[:, keep.long()].contiguous(), wf), zr.mx_quantize(X, xf, keep_idx=keep)
    Z = zr.mx_linear_fwd(X, wk, keep, DROP_K, x_fmt=xf)
    check(torch, Z, *(zr.mx_dequantize(m, torch.float32).double() for m in (xk, wk)), dtype, dtype == "bf16" and xf == E4M3)
    assert torch.equal(zr.mx_linear_fwd(xk, wk, keep, DROP_K, K=C, dtype=dt), Z)


@pytest.mark.parametrize("xf,wf", PAIRS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,C", [(1, 4096, 300), (1, 4112, 1000), (9, 4112, 7300), (16, 4099, 4200), (1, 11008, 4096), (16, 11008, 512), (3, 40000, 129)])
def test_more_columns_than_the_chip_takes_at_once(torch, zr, M, N, C, dtype, xf, wf):  # noqa: F811
    dt = tdt(torch, dtype)
    cut = dtype == "bf16" and xf == E4M3
    X, W = normal(torch, M + C, M, C, dtype=dt), normal(torch, N, N, C, dtype=dt, scale=0.05)
    wm, xm = zr.mx_quantize(W, wf), zr.mx_quantize(X, xf)
    xv, wv = (zr.mx_dequantize(m, torch.float32).double() for m in (xm, wm))
    buf = torch.full((M + 1, N + 3), 77.0, dtype=dt, device="cuda")
    Y = buf[:M, :N]
    zr.mx_linear_fwd(X, wm, Y=Y, x_fmt=xf)
    check(torch, Y, xv, wv, dtype, cut)
    assert torch.equal(zr.mx_linear_fwd(xm, wm, dtype=dt), Y)
    assert torch.all(buf[M] == 77.0) and torch.all(buf[:, N:] == 77.0)
    # kept features, the others as they were
    for n in {max(1, N - 7), N * 3 // 4}:
        s = subset(n, N, n)
        keep, k = idx(torch, s), torch.from_numpy(s).long().cuda()
        prev = normal(torch, 5, M, N + 3, dtype=dt)[:, :N]
        Z = torch.full((M + 1, N + 3), 77.0, dtype=dt, device="cuda")
        zr.mx_linear_fwd(X, wm, keep, DROP_N, SAME, prev_Y=prev, Y=Z[:M, :N], x_fmt=xf)
        check(torch, Z[:M, k], xv, wv[k], dtype, cut)
        drop = torch.ones(N, dtype=torch.bool, device="cuda")
        drop[k] = False
        assert torch.equal(Z[:M, :N][:, drop], prev[:, drop]) and torch.all(Z[M] == 77.0) and torch.all(Z[:, N:] == 77.0)
        B = zr.mx_linear_fwd(xm, wm, keep, DROP_N, dtype=dt)
        assert torch.equal(B[:, k], Z[:M, k]) and torch.all(B[:, drop] == 0)
