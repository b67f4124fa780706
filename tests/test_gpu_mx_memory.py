"""Scratch of the backward products from a checkpoint, where the binding allocates it."""
import pytest

from mx_util import E4M3
from test_gpu_mx import DROP_K, DROP_N, idx, subset
from test_gpu_mx import torch, zr  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", [DROP_K, DROP_N])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scratch_of_a_call_without_a_buffer(torch, zr, mode, dtype):  # noqa: F811
    """The checkpoint's values, and what zr_resized_linear_bwd needs beside the columns that it would extract from X: those of a
    DROP_K checkpoint are side by side already."""
    M, K, N = 40000, 776, 328              # 582 kept columns: 640 with their padding
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    n_keep = (K if mode == DROP_K else N) * 3 // 4
    held = n_keep if mode == DROP_K else K
    up64 = lambda v: (v + 63) // 64 * 64  # noqa: E731
    need = M * up64(held) * dt.itemsize + zr.workspace_bytes(M, K, N, n_keep, mode, dt)
    if mode == DROP_K and dtype == "bf16":
        need -= M * up64(n_keep) * 2
    X = zr.mx_quantize(torch.randn(M, held, device="cuda").to(dt), E4M3)
    W = torch.randn(*((K, N) if mode == DROP_K else (N, K)), device="cuda").to(dt)
    dY = torch.randn(M, N, device="cuda").to(dt)
    keep = idx(torch, subset(1, K if mode == DROP_K else N, n_keep))
    dX, dW = torch.empty(M, K, dtype=dt, device="cuda"), torch.empty_like(W)
    call = lambda ws: zr.resized_linear_bwd_mx(X, W, dY, keep, mode, dX=dX, dW=dW, workspace=ws,  # noqa: E731
                                               w_layout=0 if mode == DROP_K else 1)
    call(None)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    call(None)
    # (memory of this size comes in segments of whole 2 MiB, and a rest of up to 1 MiB stays with its block; the columns are 47 MiB)
    assert torch.cuda.max_memory_allocated() - before < need + (2 << 20)
    first = dX.clone(), dW.clone()
    call(torch.empty(need, dtype=torch.uint8, device="cuda"))
    assert torch.equal(dX, first[0]) and torch.equal(dW, first[1])
