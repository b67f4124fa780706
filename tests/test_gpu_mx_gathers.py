"""Rows into blocks by the staging kernel in each of its forms: from 1024 rows on it takes up to four to a workgroup, and rows of other
lengths take other numbers of chunks a thread.  First, last and some middle rows against the definition, byte by byte; all rows against calls
of few rows, which take one row to a workgroup."""
import numpy as np
import pytest

from mx_util import E2M1, E4M3, INT8, quantize
from test_gpu_mx import idx, same_bytes, subset, tdt
from test_gpu_mx import torch, zr  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu

# rows, bytes of a row / 2, kept (0: all, from rows off 16 bytes).  Up to 256, 512, 1024, 2048 and 4096 chunks of 16 bytes a row; where the
# rows are short, four, three and two of them to a workgroup; a last workgroup of fewer.
FORMS = [(4099, 1000, 751), (3073, 1999, 1500), (2049, 520, 0),
         (8191, 2752, 2064), (2050, 4001, 0),
         (4103, 8000, 100), (4101, 8000, 5001), (2051, 8192, 8191),
         (2053, 11008, 8256), (70, 11009, 0),
         (1500, 20000, 12001), (40, 32750, 0)]


@pytest.mark.parametrize("fmt", [E4M3, E2M1, INT8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,half,kept", FORMS)
@pytest.mark.parametrize("odd", [False, True])
def test_every_form_of_the_staging_kernel(torch, zr, rows, half, kept, dtype, fmt, odd):  # noqa: F811
    cols = half if dtype == "bf16" else half // 2
    kept = kept if dtype == "bf16" else kept // 2
    if not kept and not odd:
        kept = cols - 1                                     # (all of rows on 16 bytes have a kernel of their own)
    ld, offset = (cols + 7, 1) if odd else ((cols + 7) // 8 * 8, 0)
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    buf = torch.randn(offset + rows * ld, generator=g, device="cuda").to(tdt(torch, dtype))
    src = buf[offset:].view(rows, ld)[:, :cols]
    src.mul_(torch.exp(0.7 * torch.randn(1, cols, generator=g, device="cuda")).to(src.dtype))
    s = subset(rows, cols, kept) if kept else np.arange(cols)
    keep = idx(torch, s.astype(np.int32)) if kept else None
    pad = zr.mx_empty(rows + 1, s.size, fmt)
    pad.q.fill_(0x5a)
    pad.scales.fill_(0x5a)
    out = zr.MX(pad.q[:rows], pad.scales[:rows], s.size, fmt)
    zr.mx_quantize(src, fmt, keep_idx=keep, out=out)
    assert torch.all(pad.q[rows] == 0x5a) and torch.all(pad.scales[rows] == 0x5a)
    few = np.unique(np.r_[0:5, rows // 3, rows // 2, rows - 6:rows])
    pick = torch.from_numpy(few).cuda()
    x = src[pick].double().cpu().numpy()[:, s]
    same_bytes(zr.MX(out.q[pick], out.scales[pick], s.size, fmt), *quantize(x, fmt)[:2], fmt)
    for r in range(0, rows, 1000):
        part = zr.mx_quantize(src[r:r + 1000], fmt, keep_idx=keep)
        assert torch.equal(part.q, out.q[r:r + 1000]) and torch.equal(part.scales, out.scales[r:r + 1000]), r
