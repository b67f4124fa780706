"""Operators around a block's products, host side: sizes and every refusal of their C entry points (all before any GPU work)."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2401_11469_amd", "libzr.so")
vp, i32, i64, ci, f64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_int, ctypes.c_double, ctypes.c_size_t
NULL, SHAPE, RATIO, INDEX, DTYPE, MODE, LIMIT = 1, 2, 3, 4, 5, 6, 8
P = 0x10000         # never dereferenced: every call below fails validation first
MOST = 65535 * 32


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB):
        from paper_2401_11469_amd import build
        build.build(verbose=False)
    return ctypes.CDLL(LIB)


def call(fn, defaults, **change):
    args = dict(defaults)
    assert set(change) <= set(args), change
    args.update(change)
    return fn(*args.values())


NAN = float("nan")


def test_dropout_refusals(lib):
    fn = lib.zr_dropout
    fn.argtypes, fn.restype = [vp, i64, vp, i64, i32, i32, f64, vp, ci, vp], ci
    d = dict(x=P, ldx=64, out=P, ldo=64, rows=8, cols=64, p=0.1, rng=P, dtype=1, stream=None)
    for bad, want in ((dict(x=None), NULL), (dict(out=None), NULL), (dict(rng=None), NULL), (dict(dtype=2), DTYPE), (dict(rows=0), SHAPE),
                      (dict(cols=0), SHAPE), (dict(cols=-1), SHAPE), (dict(ldx=63), SHAPE), (dict(ldo=63), SHAPE), (dict(x=P + 1), SHAPE),
                      (dict(dtype=0, out=P + 2), SHAPE), (dict(rng=P + 4), SHAPE), (dict(rows=MOST + 1), LIMIT),
                      (dict(cols=MOST + 1, ldx=1 << 30, ldo=1 << 30), LIMIT), (dict(p=1.0), RATIO), (dict(p=-0.1), RATIO), (dict(p=NAN), RATIO)):
        assert call(fn, d, **bad) == want, bad


FWD = dict(X=P, ldx=40, W=P, ldw=64, Y=P, ldy=64, M=8, K=40, N=64, keep=P, n_keep=30, mode=1, layout=0, dtype=1, bias=P, act=4, gate=P, ldg=64,
           p=0.1, rng=P, residual=P, ldr=64, Z=P, ldz=64, ws=None, ws_bytes=0, stream=None)


def test_forward_refusals(lib):
    fn = lib.zr_resized_linear_act_fwd
    fn.argtypes = [vp, i64, vp, i64, vp, i64, i32, i32, i32, vp, i32, ci, ci, ci, vp, ci, vp, i64, f64, vp, vp, i64, vp, i64, vp, sz, vp]
    fn.restype = ci
    assert len(fn.argtypes) == len(FWD)
    for bad, want in ((dict(X=None), NULL), (dict(W=None), NULL), (dict(Y=None), NULL), (dict(rng=None), NULL), (dict(dtype=2), DTYPE),
                      (dict(mode=2), MODE), (dict(layout=2), MODE), (dict(act=5), MODE), (dict(act=-1), MODE), (dict(M=0), SHAPE), (dict(K=0), SHAPE),
                      (dict(N=0), SHAPE), (dict(M=MOST + 1), LIMIT), (dict(N=MOST + 1), LIMIT), (dict(K=MOST + 1), LIMIT), (dict(n_keep=0), INDEX),
                      (dict(n_keep=41), INDEX), (dict(mode=0, n_keep=65), INDEX), (dict(ldx=39), SHAPE), (dict(ldw=63), SHAPE),
                      (dict(layout=1, ldw=39), SHAPE), (dict(ldy=63), SHAPE), (dict(ldg=63), SHAPE), (dict(ldr=63), SHAPE), (dict(ldz=63), SHAPE),
                      (dict(p=1.0), RATIO), (dict(p=NAN), RATIO), (dict(rng=P + 1), SHAPE)):
        assert call(fn, FWD, **bad) == want, bad
    for t in ("X", "W", "Y", "bias", "gate", "residual", "Z"):
        assert call(fn, FWD, **{t: P + 1}) == SHAPE, t
        assert call(fn, FWD, **{t: P + 2}, dtype=0) == SHAPE, t


BWD = dict(X=P, ldx=40, W=P, ldw=64, dY=P, lddy=64, Z=P, ldz=64, gate=P, ldg=64, dX=P, lddx=40, dW=P, lddw=64, dbias=P, dgate=P, lddg=64,
           M=8, K=40, N=64, keep=P, n_keep=30, mode=1, layout=0, dtype=1, act=4, p=0.1, rng=P, ws=P, ws_bytes=1 << 30, stream=None)


def test_backward_refusals(lib):
    fn = lib.zr_resized_linear_act_bwd
    fn.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, i64, i32, i32, i32, vp, i32, ci, ci, ci, ci, f64, vp, vp, sz, vp]
    fn.restype = ci
    assert len(fn.argtypes) == len(BWD)
    for bad, want in ((dict(dY=None), NULL), (dict(X=None), NULL), (dict(W=None), NULL), (dict(Z=None), NULL),
                      (dict(dX=None, dW=None, dbias=None, dgate=None), NULL), (dict(act=0, Z=None), NULL),      # dgate wants Z
                      (dict(rng=None), NULL), (dict(dtype=3), DTYPE), (dict(mode=-1), MODE), (dict(layout=2), MODE), (dict(act=7), MODE),
                      (dict(M=0), SHAPE), (dict(N=MOST + 1), LIMIT), (dict(n_keep=0), INDEX), (dict(n_keep=41), INDEX), (dict(lddy=63), SHAPE),
                      (dict(ldz=63), SHAPE), (dict(ldg=63), SHAPE), (dict(lddg=63), SHAPE), (dict(lddx=39), SHAPE), (dict(lddw=63), SHAPE),
                      (dict(ldx=39), SHAPE), (dict(ldw=63), SHAPE), (dict(layout=1, ldw=39), SHAPE), (dict(p=1.5), RATIO), (dict(rng=P + 4), SHAPE),
                      (dict(ws=None), NULL), (dict(ws=P + 8), SHAPE), (dict(ws_bytes=1024), SHAPE)):
        assert call(fn, BWD, **bad) == want, bad
    # dbias alone needs room for its sums, the products room for dZ where that is not dY
    only = dict(dX=None, dW=None, dgate=None, gate=None, act=0, p=0.0)
    assert call(fn, BWD, **only, ws=None) == NULL
    assert call(fn, BWD, **only, ws_bytes=255) == SHAPE          # one slab of 64 columns
    assert call(fn, BWD, dbias=None, ws=None) == NULL
    for t in ("X", "W", "dY", "Z", "gate", "dX", "dW", "dbias", "dgate"):
        assert call(fn, BWD, **{t: P + 1}) == SHAPE, t


JOIN = dict(y=P, ldy=64, x=P, ldx=64, x_out=P, ldxo=64, h=P, ldh=64, rows=8, cols=64, norms=3, norm=0, eps=1e-5, p=0.1, rng=P, scale=1.0,
            bias=P, gate=P, post_w=P, post_b=P, pre_w=P, pre_b=P, dtype=1, stream=None)
SHARED = ((dict(dtype=2), DTYPE), (dict(norms=4), MODE), (dict(norms=-1), MODE), (dict(norm=2), MODE), (dict(rows=0), SHAPE), (dict(cols=0), SHAPE),
          (dict(rows=MOST + 1), LIMIT), (dict(cols=16385), LIMIT), (dict(eps=-1.0), RATIO), (dict(eps=NAN), RATIO), (dict(p=1.0), RATIO),
          (dict(rng=None), NULL), (dict(rng=P + 2), SHAPE))


def test_join_refusals(lib):
    fn = lib.zr_block_join_fwd
    fn.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, i32, i32, ci, ci, f64, f64, vp, f64, vp, vp, vp, vp, vp, vp, ci, vp]
    fn.restype = ci
    assert len(fn.argtypes) == len(JOIN)
    for bad, want in SHARED + ((dict(y=None), NULL), (dict(x=None), NULL), (dict(x_out=None), NULL), (dict(h=None), NULL), (dict(ldy=63), SHAPE),
                               (dict(ldx=63), SHAPE), (dict(ldxo=63), SHAPE), (dict(ldh=63), SHAPE)):
        assert call(fn, JOIN, **bad) == want, bad
    for t in ("y", "x", "x_out", "h", "bias", "gate", "post_w", "post_b", "pre_w", "pre_b"):
        assert call(fn, JOIN, **{t: P + 1}) == SHAPE, t


BACK = dict(dx_out=P, lddxo=64, dh=P, lddh=64, x_out=P, ldxo=64, y=P, ldy=64, dx=P, lddx=64, dy=P, lddy=64, rows=8, cols=64, norms=3, norm=1,
            eps=1e-5, p=0.1, rng=P, scale=1.0, bias=P, gate=P, post_w=P, post_b=P, pre_w=P, dbias=P, dgate=P, dpost_w=P, dpost_b=P, dpre_w=P,
            dpre_b=P, ws=P, ws_bytes=1 << 30, dtype=1, stream=None)


def test_join_backward_refusals(lib):
    fn = lib.zr_block_join_bwd
    fn.argtypes = [vp, i64] * 6 + [i32, i32, ci, ci, f64, f64, vp, f64] + [vp] * 11 + [vp, sz, ci, vp]
    fn.restype = ci
    assert len(fn.argtypes) == len(BACK)
    none = {n: None for n in ("dx", "dy", "dbias", "dgate", "dpost_w", "dpost_b", "dpre_w", "dpre_b")}
    for bad, want in SHARED + ((none, NULL), (dict(dh=None), NULL), (dict(x_out=None), NULL), (dict(y=None), NULL),
                               (dict(norms=0, dx_out=None, dpost_w=None, dpost_b=None, dpre_w=None, dpre_b=None), NULL),
                               (dict(norms=1), MODE), (dict(norms=2), MODE), (dict(norms=2, dpost_w=None), MODE),
                               (dict(norms=2, dpost_w=None, dpost_b=None, y=None), NULL),          # dgate wants y
                               (dict(lddxo=63), SHAPE), (dict(lddh=63), SHAPE), (dict(ldxo=63), SHAPE), (dict(ldy=63), SHAPE), (dict(lddx=63), SHAPE),
                               (dict(lddy=63), SHAPE), (dict(ws=None), NULL), (dict(ws=P + 8), SHAPE), (dict(ws_bytes=6 * 64 * 4 - 1), SHAPE)):
        assert call(fn, BACK, **bad) == want, bad
    for t in ("dx_out", "dh", "x_out", "y", "dx", "dy", "bias", "gate", "post_w", "post_b", "pre_w", "dbias", "dgate", "dpost_w", "dpost_b",
              "dpre_w", "dpre_b"):
        assert call(fn, BACK, **{t: P + 1}) == SHAPE, t


def test_sizes(lib):
    f, b, j = lib.zr_act_fwd_workspace_bytes, lib.zr_act_bwd_workspace_bytes, lib.zr_block_join_workspace_bytes
    for fn in (f, b):
        fn.argtypes, fn.restype = [i32, i32, i32, i32, ci, ci], sz
    j.argtypes, j.restype = [i32, i32], sz
    plain = lib.zr_workspace_bytes
    plain.argtypes, plain.restype = [i32] * 4 + [ci, ci], sz
    assert f(0, 1, 1, 1, 0, 1) == 0 and f(1, 1, 1, 1, 0, 2) == 0 and f(8, 0, 8, 8, 0, 1) == 0 and f(8, 8, 8, 0, 0, 1) == 0
    assert f(100, 300, 200, 250, 1, 1) >= 100 * 256 * 2                          # the kept columns of X, rounded up to 64
    for dt, size in ((0, 4), (1, 2)):
        assert b(100, 300, 201, 250, 1, dt) >= 100 * 208 * size + 201 * 4 + plain(100, 300, 201, 250, 1, dt)
        assert b(0, 300, 201, 250, 1, dt) == 0
    assert b(1 << 20, 1 << 13, 1 << 16, 1 << 13, 0, 1) > (1 << 37)              # (no 32 bits on the way)
    assert j(0, 8) == 0 and j(8, 0) == 0 and j(8, 16385) == 0 and j(1, 8) >= 5 * 8 * 4 and j(1 << 20, 16384) >= 5 * 16384 * 4

