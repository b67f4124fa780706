"""The operators around a block's products in 64 bits, from their definitions, on the CPU, and how far a GPU result may be off.

Bounds.  u: half a step of the output type relative to the value (bf16 2^-8, fp32 2^-24), for the one rounding of a result.
f = 2^-24: half a step of the fp32 arithmetic between.  A sum of C fp32 products is off by 8 sqrt(C) f times the root of the sum of
their squares (a random walk of its roundings, eight standard deviations and more), as for the resized products.
"""
import numpy as np
from scipy import special

NONE, RELU, GELU, GELU_TANH, SILU = range(5)
RMS, LAYER = 0, 1
F = 2.0 ** -24
U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def philox(counter, key, rounds=7):
    """Philox 4 x 32 (Salmon, Moraes, Dror and Shaw 2011) in Python integers."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def halves(seed, offset, rows, cols, first_row=0):
    """[rows, cols]: the 16 bits that each element looks at."""
    u = np.uint64
    groups = -(-cols // 8)
    low, w = u(0xFFFFFFFF), u(32)
    c = [np.broadcast_to(v, (rows, groups)) for v in (np.arange(groups, dtype=u)[None], np.arange(first_row, first_row + rows, dtype=u)[:, None],
                                                      u(offset & 0xFFFFFFFF), u(offset >> 32))]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(7):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(b >> w) ^ c[1] ^ u(k0), b & low, (a >> w) ^ c[3] ^ u(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = np.stack(c, axis=-1)
    return np.stack([words & u(0xFFFF), words >> u(16)], axis=-1).reshape(rows, -1)[:, :cols].astype(np.int64)


def factor(seed, offset, rows, cols, p):
    q = min(65535, int(np.floor(p * 65536 + 0.5)))
    if q == 0:
        return np.ones((rows, cols))
    return np.where(halves(seed, offset, rows, cols) >= q, 65536.0 / (65536 - q), 0.0)


def times(f, x):
    """f * x, 0 where f is, whatever x is there."""
    return np.where(f == 0, 0.0, f * np.where(f == 0, 0.0, x))


def act(kind, z):
    """(value, slope)"""
    one = np.ones_like(z)
    if kind == RELU:
        return np.where(z > 0, z, 0.0), np.where(z > 0, 1.0, 0.0)
    if kind == GELU:
        cdf = special.erfc(-z / np.sqrt(2.0)) / 2
        return z * cdf, cdf + z * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
    if kind == GELU_TANH:
        b = np.sqrt(2 / np.pi)
        t = special.expit(2 * b * (z + 0.044715 * z ** 3))
        return z * t, t + z * t * (1 - t) * 2 * b * (1 + 3 * 0.044715 * z * z)
    if kind == SILU:
        t = special.expit(z)
        return z * t, t + z * t * (1 - t)
    return z, one


def act_error(kind, z, a):
    """How far the value and the slope may be off for an exact z.  Their exponential has an argument of w = |z|, z^2 / 2 or
    1.6 |z| + 0.07 |z|^3, which is off by 3 f w, so the exponential by (3 w + 3) f of itself and what it makes of it by
    (3 w + 12) f; gelu in bf16 uses a formula that is off by 0.75e-7 in its distribution function; |slope| <= 1.2."""
    if kind in (NONE, RELU):
        return np.zeros_like(z), np.zeros_like(z)
    w = {GELU: z * z / 2, GELU_TANH: 1.6 * abs(z) + 0.072 * abs(z) ** 3, SILU: abs(z)}[kind]
    rel = (3 * w + 12) * F
    # (the exponential's share of value and slope never exceeds 1.2 and falls as e^-w: w e^-w <= 0.37)
    return rel * abs(a) + 1.5e-7 * abs(z), 1.2 * 16 * F * (1 + z * z) + 1.5e-7 * (1 + z * z)


def spread(kept, n, axis, keep):
    shape = list(kept.shape)
    shape[axis] = n
    out = np.zeros(shape)
    if axis == 0:
        out[keep] = kept
    else:
        out[:, keep] = kept
    return out


def product(X, W, keep, mode_k, bias, kind, gate, f, residual, dtype):
    """W [K, N].  ((Y, bound), (Z, bound))"""
    u = U[dtype]
    if mode_k:
        z, l2 = X[:, keep] @ W[keep], np.sqrt(X[:, keep] ** 2 @ W[keep] ** 2)
    else:
        N = W.shape[1]
        z, l2 = spread(X @ W[:, keep], N, 1, keep), spread(np.sqrt(X ** 2 @ W[:, keep] ** 2), N, 1, keep)
    C = len(keep) if mode_k else X.shape[1]
    ez = 8 * np.sqrt(C) * F * l2
    if bias is not None:
        z = z + bias
        ez = ez + F * abs(z)
    a, _ = act(kind, z)
    ea = 1.2 * ez + act_error(kind, z, a)[0]
    g = 1.0 if gate is None else gate
    t = times(f, a * g)
    r = 0.0 if residual is None else residual
    y = t + r
    ey = f * abs(g) * ea + 4 * F * abs(t) + F * abs(y) + u * abs(y) * (1 + 2.0 ** -10) + 1e-37
    return (y, ey * 1.01), (z, (ez + u * abs(z) * (1 + 2.0 ** -10) + 1e-37) * 1.01)


def product_back(X, W, dY, Z, keep, mode_k, kind, gate, f, dtype):
    """(dX, dW [K, N], dbias, dgate), each with its bound.  dZ is rounded once more before the products: u / sqrt(3) of a term at
    random, five times the root of the sum of the squares is more than eight standard deviations."""
    u = U[dtype]
    uz = u if dtype == "bf16" else 0.0
    a, s = act(kind, Z)
    ea, es = act_error(kind, Z, a)
    t = times(f, dY)
    g = 1.0 if gate is None else gate
    dz = t * g * s
    edz = abs(t * g) * es + 4 * F * abs(dz)
    dg, edg = t * a, abs(t) * ea + 3 * F * abs(t * a)
    if mode_k:
        w = W[keep]
        dX, dW = spread(dz @ w.T, W.shape[0], 1, keep), spread(X[:, keep].T @ dz, W.shape[0], 0, keep)
        lx = spread(np.sqrt(dz ** 2 @ w.T ** 2), W.shape[0], 1, keep)
        lw = spread(np.sqrt(X[:, keep].T ** 2 @ dz ** 2), W.shape[0], 0, keep)
        ex, ew = spread(edz @ abs(w.T), W.shape[0], 1, keep), spread(abs(X[:, keep].T) @ edz, W.shape[0], 0, keep)
        cx = W.shape[1]
    else:
        d, e, w = dz[:, keep], edz[:, keep], W[:, keep]
        dX, lx, ex = d @ w.T, np.sqrt(d ** 2 @ w.T ** 2), e @ abs(w.T)
        dW, lw, ew = (spread(v, W.shape[1], 1, keep) for v in (X.T @ d, np.sqrt(X.T ** 2 @ d ** 2), abs(X.T) @ e))
        cx = len(keep)
    M = X.shape[0]
    done = lambda v, e: (v, (e + u * abs(v) * (1 + 2.0 ** -10) + 1e-37) * 1.01)      # noqa: E731
    db = dz.sum(axis=0)
    return (done(dX, ex + (5 * uz + 8 * np.sqrt(cx) * F) * lx), done(dW, ew + (5 * uz + 8 * np.sqrt(M) * F) * lw),
            done(db, edz.sum(axis=0) + 8 * np.sqrt(M) * F * np.sqrt((dz ** 2).sum(axis=0))), done(dg, edg))


def norm(v, kind, eps):
    if kind == LAYER:
        v = v - v.mean(axis=1, keepdims=True)
    r = 1 / np.sqrt((v * v).mean(axis=1, keepdims=True) + eps)
    return v * r, r


def _vec(v, other):
    return other if v is None else v


def join(y, x, kind, post, pre, eps, f, scale, vec, dtype):
    """(x_out, bound), (h, bound).  A norm's mean and deviation come from sums of n terms in fp32, a tree of a few levels over 16 in
    a row, and a square root and a division: (n's tree) 32 f of the row's largest value covers each of them."""
    u = U[dtype]
    t = times(f, y + _vec(vec.get("bias"), 0.0))
    et = 3 * F * abs(t)
    n, en = t, et
    if post:
        hat, r = norm(t, kind, eps)
        w, b = _vec(vec.get("post_w"), 1.0), _vec(vec.get("post_b"), 0.0)
        n = hat * w + b
        # (a shift by the mean leaves an error of the size of what was there before it)
        en = abs(w) * 32 * F * (abs(hat) + r * abs(t).max(axis=1, keepdims=True)) + 2 * F * abs(n)
    g = scale * _vec(vec.get("gate"), 1.0)
    xo = x + g * n
    ex = abs(g) * en + 3 * F * abs(g * n) + F * abs(xo)
    out = [(xo, (ex + u * abs(xo) * (1 + 2.0 ** -10) + 1e-37) * 1.01)]
    if pre:
        hat, r = norm(xo, kind, eps)
        w, b = _vec(vec.get("pre_w"), 1.0), _vec(vec.get("pre_b"), 0.0)
        h = hat * w + b
        largest = abs(xo).max(axis=1, keepdims=True)
        eh = abs(w) * (r * (ex + ex.max(axis=1, keepdims=True) * (1 + abs(hat))) + 32 * F * (abs(hat) + r * largest)) + 2 * F * abs(h)
        out.append((h, (eh + u * abs(h) * (1 + 2.0 ** -10) + 1e-37) * 1.01))
    return out


def norm_back(g, hat, r, kind):
    d = g - hat * (g * hat).mean(axis=1, keepdims=True)
    if kind == LAYER:
        d = d - g.mean(axis=1, keepdims=True)
    return d * r


def unjoin(dxo, dh, xo, y, kind, post, pre, eps, f, scale, vec, dtype):
    """dict of (value, bound): dx, dy and the vectors'.  An element of a norm's gradient is off by 64 f of the largest sum of its
    terms' sizes in its row (each term: a normalised value, a mean over the row, a few products), and by what its own g is off."""
    u = U[dtype]
    out = {}

    def sums(v, e):
        return v.sum(axis=0), e.sum(axis=0) + 8 * np.sqrt(len(v)) * F * np.sqrt((v * v).sum(axis=0))

    def back(g, eg, v):
        hat, r = norm(v, kind, eps)
        off = 32 * F * (1 + r * abs(v).max(axis=1, keepdims=True))        # of hat
        size = r * (abs(g) + abs(g).mean(axis=1, keepdims=True) + (1 + abs(hat)) * abs(g * hat).mean(axis=1, keepdims=True))
        e = 2 * off * size.max(axis=1, keepdims=True) + r * (eg + eg.mean(axis=1, keepdims=True) + abs(hat) * (eg * abs(hat)).mean(axis=1, keepdims=True))
        return hat, off, norm_back(g, hat, r, kind), e

    dx = np.zeros_like(dxo if dxo is not None else dh) + (0.0 if dxo is None else dxo)
    ex = np.zeros_like(dx)
    if pre:
        g = dh * _vec(vec.get("pre_w"), 1.0)
        hat, off, d, e = back(g, 2 * F * abs(g), xo)
        dx, ex = dx + d, e + F * abs(dx)
        out["pre_w"] = sums(dh * hat, abs(dh) * off * (1 + abs(hat)))
        out["pre_b"] = sums(dh, 0 * dh)
    out["dx"] = dx, ex
    s = scale * dx
    es = abs(scale) * ex + 2 * F * abs(s)
    t = None if y is None else times(f, y + _vec(vec.get("bias"), 0.0))
    if post:
        hat_t, r_t = norm(t, kind, eps)
        off_t = 32 * F * (1 + r_t * abs(t).max(axis=1, keepdims=True))
        n = hat_t * _vec(vec.get("post_w"), 1.0) + _vec(vec.get("post_b"), 0.0)
        en = abs(_vec(vec.get("post_w"), 1.0)) * off_t * (1 + abs(hat_t)) + 2 * F * abs(n)
    else:
        n, en = t, None if t is None else 3 * F * abs(t)
    if n is not None:
        out["gate"] = sums(s * n, abs(s) * en + es * abs(n) + F * abs(s * n))
    dn = s * _vec(vec.get("gate"), 1.0)
    en_ = es * abs(_vec(vec.get("gate"), 1.0)) + F * abs(dn)
    if post:
        out["post_w"] = sums(dn * hat_t, abs(dn) * off_t * (1 + abs(hat_t)) + en_ * abs(hat_t))
        out["post_b"] = sums(dn, en_)
        w = _vec(vec.get("post_w"), 1.0)
        _, _, dn, en_ = back(dn * w, en_ * abs(w) + F * abs(dn * w), t)
    dy = times(f, dn)
    ey = f * en_ + 2 * F * abs(dy)
    out["dy"] = dy, ey
    out["bias"] = sums(dy, ey)
    return {k: (v, (e + u * abs(v) * (1 + 2.0 ** -10) + 1e-37) * 1.01) for k, (v, e) in out.items()}
