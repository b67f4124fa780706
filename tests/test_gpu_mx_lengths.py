"""Block-scaled operators at the far end of the sizes, where the lanes of one launch would pass 32 bits."""
import pytest

from mx_util import E2M1
from test_gpu_mx import torch, zr  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


def test_long_rows_beyond_32_bits_of_threads(torch, zr):  # noqa: F811
    """Gathered rows that are staged nowhere, a wavefront for 512 values: 1.1 M x 32759 of them are 4.5 G lanes."""
    rows, cols = 1_100_000, 32760
    if torch.cuda.mem_get_info()[0] < 110 << 30:
        pytest.skip("needs 110 GB of memory")
    src = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    keep = torch.arange(1, cols, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    picked = [slice(0, 3), slice(rows // 2, rows // 2 + 3), slice(rows - 3, rows)]
    for p in picked:
        src[p] = torch.randn(3, cols, generator=g, device="cuda").bfloat16()
    out = zr.mx_empty(rows, cols - 1, E2M1)
    for p in picked:
        out.q[p] = 0x55
        out.scales[p] = 0x55
    zr.mx_quantize(src, E2M1, keep_idx=keep, out=out)
    for p in picked:
        part = zr.mx_quantize(src[p], E2M1, keep_idx=keep)
        assert torch.equal(out.q[p], part.q) and torch.equal(out.scales[p], part.scales), p
    del src, out
    torch.cuda.empty_cache()


def test_product_beyond_32_bits_of_threads(torch, zr):  # noqa: F811
    """A short contraction runs on tiles of 64 x 64 on 256 lanes: 2097120 x 32800 results are 16.8 M of them."""
    M, K, N = 65535 * 32, 32, 32800
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("needs 150 GB of memory")
    g = torch.Generator(device="cuda").manual_seed(2)
    X = zr.mx_quantize(torch.randn(M, K, generator=g, device="cuda").bfloat16(), E2M1)
    W = zr.mx_quantize(torch.randn(N, K, generator=g, device="cuda").bfloat16(), E2M1)
    Y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    picked = [slice(0, 40), slice(M // 2, M // 2 + 40), slice(M - 40, M)]
    for p in picked:
        Y[p] = 77.0
    zr.mx_linear_fwd(X, W, Y=Y)
    for p in picked:
        part = zr.mx_linear_fwd(zr.MX(X.q[p], X.scales[p], K, E2M1), W)     # (one instruction deep: no order of sums)
        assert torch.equal(Y[p], part), p
    del Y
    torch.cuda.empty_cache()
