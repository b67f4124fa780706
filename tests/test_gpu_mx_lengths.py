"""Into blocks at the far end of the sizes: more rows of more values than one thread each could be launched for."""
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
