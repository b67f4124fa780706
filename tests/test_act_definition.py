"""The definitions that the tests of the operators around a block's products compare with: the generator against its authors'
published outputs, slopes and gradients against differences, in 64 bits on the CPU."""
import numpy as np
import pytest

import act_util as au


@pytest.mark.parametrize("rounds,counter,key,want", [
    (7, 0, 0, "5f6fb709 0d893f64 4f121f81 4f730a48"),
    (10, 0, 0, "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
])
def test_generator_gives_its_authors_outputs(rounds, counter, key, want):
    assert " ".join(f"{v:08x}" for v in au.philox([counter] * 4, [key] * 2, rounds)) == want


def test_halves_are_the_words_of_one_call():
    seed, offset = 0x123456789ABCDEF0, 0xFEDCBA9876543210
    h = au.halves(seed, offset, 5, 21)
    for r, c in ((0, 0), (3, 7), (4, 8), (2, 20)):
        w = au.philox([c // 8, r, offset & 0xFFFFFFFF, offset >> 32], [seed & 0xFFFFFFFF, seed >> 32])[c % 8 // 2]
        assert h[r, c] == (w >> 16 if c % 2 else w & 0xFFFF)


def test_dropped_share_and_mean():
    f = au.factor(5, 6, 512, 512, 0.1)
    n = f.size
    # binomial: five standard deviations
    assert abs((f == 0).mean() - 0.1) < 5 * np.sqrt(0.09 / n) + 2.0 ** -17
    assert abs(f.mean() - 1) < 5 * np.sqrt(0.1 / 0.9 / n)
    assert len(np.unique(f)) == 2


@pytest.mark.parametrize("kind", range(5))
def test_slopes_against_differences(kind):
    z = np.linspace(-6, 6, 241) + 0.0123                      # (no point at the kink of relu)
    h = 1e-5
    slope = (au.act(kind, z + h)[0] - au.act(kind, z - h)[0]) / (2 * h)
    # the third derivative is below 3: h^2 / 6 of it, and the roundings over h
    np.testing.assert_allclose(au.act(kind, z)[1], slope, rtol=0, atol=h * h + 1e-10)


@pytest.mark.parametrize("mode_k", [False, True])
def test_product_gradients_against_differences(mode_k):
    g = np.random.default_rng(3)
    M, K, N = 5, 7, 6
    X, W, b, G, R, dY = (g.standard_normal(s) for s in ((M, K), (K, N), N, (M, N), (M, N), (M, N)))
    keep = np.array([0, 2, 3, 5])
    f = au.factor(9, 1, M, N, 0.3)

    def loss(X, W, b, G):
        (y, _), _ = au.product(X, W, keep, mode_k, b, au.SILU, G, f, R, "f32")
        return (y * dY).sum()

    _, (Z, _) = au.product(X, W, keep, mode_k, b, au.SILU, G, f, R, "f32")
    dX, dW, db, dG = (v for v, _ in au.product_back(X, W, dY, Z, keep, mode_k, au.SILU, G, f, "f32"))
    for i, d in enumerate((dX, dW, db, dG)):
        v = g.standard_normal(d.shape)
        args = [X, W, b, G]
        h = 1e-5
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + h * v, args[i] - h * v
        got = (loss(*up) - loss(*down)) / (2 * h)
        want = (d * v).sum()
        # (the zeros of the pruned slices too: those do not enter the product)
        assert abs(got - want) < 1e-7 * (1 + abs(want))


@pytest.mark.parametrize("kind", [au.RMS, au.LAYER])
@pytest.mark.parametrize("post,pre", [(False, False), (True, False), (False, True), (True, True)])
def test_join_gradients_against_differences(kind, post, pre):
    g = np.random.default_rng(4)
    R, C, scale, eps = 4, 9, 0.7, 1e-5
    names = ["y", "x", "bias", "gate"] + ["post_w", "post_b"] * post + ["pre_w", "pre_b"] * pre
    args = {n: g.standard_normal((R, C) if n in ("y", "x") else C) for n in names}
    wx, wh = g.standard_normal((R, C)), g.standard_normal((R, C))
    f = au.factor(2, 3, R, C, 0.25)

    def forward(a):
        return au.join(a["y"], a["x"], kind, post, pre, eps, f, scale, a, "f32")

    def loss(a):
        out = forward(a)
        return (out[0][0] * wx).sum() + ((out[1][0] * wh).sum() if pre else 0)

    xo = forward(args)[0][0]
    grads = au.unjoin(wx, wh if pre else None, xo, args["y"], kind, post, pre, eps, f, scale, args, "f32")
    for n in names:
        d = grads[{"y": "dy", "x": "dx"}.get(n, n)][0]
        v = g.standard_normal(d.shape)
        h = 1e-5
        got = (loss({**args, n: args[n] + h * v}) - loss({**args, n: args[n] - h * v})) / (2 * h)
        want = (d * v).sum()
        assert abs(got - want) < 1e-7 * (1 + abs(want)), n
