"""Block-scaled operators, host side: sizes, and every refusal of their C entry points (all before any GPU work), and of
the Python binding."""
import ctypes
import os

import pytest

from mx_util import E2M1, E4M3, INT8

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2401_11469_amd", "libzr.so")
vp, i32, i64, ci = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_int
NULL, SHAPE, INDEX, DTYPE, MODE, POLICY, LIMIT = 1, 2, 4, 5, 6, 7, 8
P = 0x10000         # never dereferenced: every call below fails validation first


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB):
        from paper_2401_11469_amd import build
        build.build(verbose=False)
    return ctypes.CDLL(LIB)


def test_sizes(lib):
    rb, sb, ws = lib.zr_mx_row_bytes, lib.zr_mx_scale_bytes, lib.zr_mx_bwd_workspace_bytes
    rb.argtypes, sb.argtypes, ws.argtypes = [i32, ci], [i32], [i32, i32, i32, i32, ci, ci]
    rb.restype = sb.restype = ws.restype = ctypes.c_size_t
    assert [rb(n, E4M3) for n in (1, 128, 129, 2064)] == [128, 128, 256, 2176]
    assert [rb(n, E2M1) for n in (1, 128, 129, 2064)] == [64, 64, 128, 1088]
    assert rb(129, INT8) == 256 and rb(0, E4M3) == 0 and rb(5, 3) == 0 and rb(5, -1) == 0
    assert [sb(n) for n in (0, 1, 512, 513, 2048)] == [0, 16, 16, 32, 64]
    plain = lib.zr_workspace_bytes
    plain.argtypes, plain.restype = [i32] * 4 + [ci, ci], ctypes.c_size_t
    assert ws(100, 300, 200, 250, 1, 1) == 100 * 256 * 2 + plain(100, 300, 200, 250, 1, 1)     # DROP_K: the kept columns
    assert ws(100, 300, 200, 150, 0, 0) == 100 * 320 * 4 + plain(100, 300, 200, 150, 0, 0)     # DROP_N: all of X
    assert ws(0, 300, 200, 150, 0, 0) == 0 and ws(100, 300, 200, 150, 0, 7) == 0


def test_largest_sizes_do_not_wrap(lib):
    rb, sb = lib.zr_mx_row_bytes, lib.zr_mx_scale_bytes
    rb.argtypes, sb.argtypes = [i32, ci], [i32]
    rb.restype = sb.restype = ctypes.c_size_t
    assert rb(2 ** 31 - 1, E4M3) == 2 ** 31 and sb(2 ** 31 - 1) == 2 ** 26


def call(fn, defaults, **change):
    args = dict(defaults)
    assert set(change) <= set(args), change
    args.update(change)
    return fn(*args.values())


def test_quantize_refusals(lib):
    fn = lib.zr_mx_quantize
    fn.argtypes, fn.restype = [vp, i64, i32, i32, ci, vp, i32, ci, ci, vp, i64, vp, i64, vp], ci
    d = dict(src=P, ld=64, rows=8, cols=64, axis=1, keep=P, n_keep=40, dtype=1, fmt=E4M3, q=P, ldq=128, s=P, lds=16, stream=None)
    for bad, want in ((dict(src=None), NULL), (dict(q=None), NULL), (dict(s=None), NULL), (dict(dtype=2), DTYPE), (dict(fmt=3), DTYPE),
                      (dict(fmt=-1), DTYPE), (dict(rows=0), SHAPE), (dict(cols=0), SHAPE), (dict(ld=63), SHAPE), (dict(axis=2), SHAPE),
                      (dict(src=P + 1), SHAPE), (dict(dtype=0, src=P + 2), SHAPE), (dict(rows=65535 * 32 + 1), LIMIT),
                      (dict(cols=65535 * 32 + 1, ld=1 << 30), LIMIT), (dict(n_keep=0), INDEX), (dict(n_keep=65), INDEX),
                      (dict(axis=0, n_keep=9), INDEX), (dict(ldq=112), SHAPE), (dict(ldq=136), SHAPE), (dict(q=P + 8), SHAPE),
                      (dict(s=P + 4), SHAPE), (dict(lds=8), SHAPE), (dict(lds=24), SHAPE), (dict(lds=0), SHAPE)):
        assert call(fn, d, **bad) == want, bad
    # without a list the whole axis has to fit
    assert call(fn, d, keep=None, n_keep=0, cols=200, ld=200) == SHAPE
    assert call(fn, d, keep=None, n_keep=-5, cols=129, ld=130) == SHAPE


def test_dequantize_refusals(lib):
    fn = lib.zr_mx_dequantize
    fn.argtypes, fn.restype = [vp, i64, vp, i64, i32, i32, ci, vp, i64, ci, vp], ci
    d = dict(q=P, ldq=128, s=P, lds=16, rows=8, n=100, fmt=E4M3, out=P, ldo=100, dtype=1, stream=None)
    for bad, want in ((dict(q=None), NULL), (dict(s=None), NULL), (dict(out=None), NULL), (dict(fmt=7), DTYPE), (dict(dtype=-1), DTYPE),
                      (dict(rows=0), SHAPE), (dict(n=0), SHAPE), (dict(ldo=99), SHAPE), (dict(n=129, ldo=200), SHAPE), (dict(ldq=64), SHAPE),
                      (dict(lds=0), SHAPE), (dict(q=P + 1), SHAPE), (dict(s=P + 8), SHAPE), (dict(out=P + 1), SHAPE),
                      (dict(out=P + 2, dtype=0), SHAPE), (dict(rows=65535 * 32 + 1), LIMIT)):
        assert call(fn, d, **bad) == want, bad


def test_product_refusals(lib):
    fn = lib.zr_mx_linear_fwd
    fn.argtypes = [vp, i64, vp, i64, vp, i64, ci, vp, i64, vp, i64, ci, vp, i64, i32, i32, i32, vp, i32, ci, ci, ci, vp, vp]
    fn.restype = ci
    d = dict(X=P, ldx=256, Xq=P, ldxq=256, Xs=P, ldxs=16, x_fmt=E4M3, Wq=P, ldwq=128, Ws=P, ldws=16, w_fmt=E2M1, Y=P, ldy=96,
             M=32, K=256, N=96, keep=P, n_keep=64, mode=0, dtype=1, policy=0, prev=None, stream=None)
    for bad, want in ((dict(Wq=None), NULL), (dict(Ws=None), NULL), (dict(Y=None), NULL), (dict(X=None, Xq=None, Xs=None), NULL),
                      (dict(Xq=None), NULL), (dict(Xs=None), NULL), (dict(Xq=None, Xs=None), NULL),           # 32 rows without a place
                      (dict(Xq=None, Xs=None, M=17), NULL), (dict(dtype=3), DTYPE), (dict(x_fmt=INT8), DTYPE), (dict(w_fmt=INT8), DTYPE),
                      (dict(x_fmt=E2M1, w_fmt=E4M3), DTYPE), (dict(x_fmt=9), DTYPE), (dict(mode=2), MODE), (dict(policy=3), POLICY),
                      (dict(policy=2), POLICY), (dict(M=0), SHAPE), (dict(K=0), SHAPE), (dict(N=0), SHAPE), (dict(ldy=95), SHAPE),
                      (dict(ldx=255), SHAPE), (dict(n_keep=97), INDEX), (dict(n_keep=0), INDEX), (dict(mode=1, n_keep=257), INDEX),
                      (dict(ldwq=64), SHAPE), (dict(ldws=0), SHAPE), (dict(ldxq=128), SHAPE), (dict(ldxs=0), SHAPE), (dict(Wq=P + 8), SHAPE),
                      (dict(X=P + 1), SHAPE), (dict(Y=P + 1), SHAPE), (dict(M=65535 * 32 + 1), LIMIT), (dict(N=65535 * 32 + 1, ldy=1 << 30), LIMIT)):
        assert call(fn, d, **bad) == want, bad
    # DROP_K: the operands hold n_keep values a row
    assert call(fn, d, mode=1, n_keep=129, ldxq=256, ldwq=64) == SHAPE
    assert call(fn, d, mode=1, n_keep=129, ldxq=128, ldwq=128) == SHAPE


def test_backward_refusals(lib):
    fn = lib.zr_resized_linear_bwd_mx
    fn.argtypes = [vp, i64, vp, i64, ci, vp, i64, vp, i64, vp, i64, vp, i64, i32, i32, i32, vp, i32, ci, ci, ci, ci, vp, vp, vp,
                   ctypes.c_size_t, vp]
    fn.restype = ci
    d = dict(Xq=P, ldxq=256, Xs=P, ldxs=16, x_fmt=E4M3, W=P, ldw=96, dY=P, lddy=96, dX=P, lddx=200, dW=P, lddw=96, M=32, K=200, N=96,
             keep=P, n_keep=150, mode=1, layout=0, dtype=1, policy=0, prev_dX=None, prev_dW=None, ws=P, ws_bytes=32 * 192 * 2, stream=None)
    for bad, want in ((dict(Xq=None), NULL), (dict(Xs=None), NULL), (dict(W=None), NULL), (dict(dY=None), NULL), (dict(dX=None, dW=None), NULL),
                      (dict(keep=None), NULL), (dict(ws=None), NULL), (dict(ws_bytes=32 * 192 * 2 - 1), SHAPE), (dict(ws=P + 8), SHAPE),
                      (dict(ws_bytes=0), SHAPE), (dict(x_fmt=3), DTYPE), (dict(dtype=5), DTYPE), (dict(mode=4), MODE), (dict(layout=2), MODE),
                      (dict(policy=5), POLICY), (dict(policy=2), POLICY), (dict(n_keep=201), INDEX), (dict(n_keep=0), INDEX), (dict(M=0), SHAPE),
                      (dict(ldw=95), SHAPE), (dict(lddy=95), SHAPE), (dict(lddx=199), SHAPE), (dict(lddw=95), SHAPE), (dict(ldxq=128), SHAPE),
                      (dict(ldxs=8), SHAPE), (dict(Xq=P + 4), SHAPE), (dict(M=65535 * 32 + 1), LIMIT)):
        assert call(fn, d, **bad) == want, bad


def test_binding_refuses_tensors_elsewhere():
    import torch
    from paper_2401_11469_amd import zr
    if torch.cuda.is_available():
        pytest.skip("looks at what the binding says without a GPU")
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    m = zr.mx_empty(4, 64, zr.MX_E4M3, device="cpu")
    assert m.q.shape == (4, 128) and m.scales.shape == (4, 16)
    for f in (lambda: zr.mx_quantize(x, zr.MX_E4M3), lambda: zr.mx_dequantize(m), lambda: zr.mx_linear_fwd(x, m)):
        with pytest.raises((ValueError, RuntimeError, AssertionError)):
            f()


def test_binding_refuses_empty_lists_and_narrow_storage():
    """What the binding looks at before any pointer is used (a device index of -1 is the CPU's)."""
    import torch
    from paper_2401_11469_amd import zr
    with pytest.raises(zr.ZrError):
        zr._list(torch.empty(0, dtype=torch.int32), -1)
    assert zr._list(None, -1) == (None, 0) and zr._list(torch.zeros(3, dtype=torch.int32), -1)[1] == 3
    wide = torch.empty(4, 4096, dtype=torch.uint8)
    for fmt, row in ((zr.MX_E4M3, 384), (zr.MX_INT8, 384), (zr.MX_E2M1, 192)):
        good = zr.MX(wide[:, :row], wide[:, :16], 300, fmt)
        assert zr._mx(good, 4, 300, -1, "m")[1::2] == (4096, 4096)
        for bad in (good._replace(q=wide[:, :row - 1]), good._replace(scales=wide[:, :15]), good._replace(n=385),
                    zr.MX(wide, wide[:, :16], 513, fmt)):
            with pytest.raises(ValueError):
                zr._mx(bad, 4, bad.n, -1, "m")
