"""What stands around the products of a block's linear layers, as cases that can be timed and checked.

  product   Y = R + D(act(X W + bias) * G): the (resized) product with bias, activation, gate, dropout and residual.
  backward  the gradients of that: of X, W, the bias and the gate.
  dropout   D(x): elements dropped by a counter-based generator; there is no mask.
  join      a block's output joins the residual stream and the next block's input leaves it:
            x' = x + scale * gate * post(D(y + bias)), h = pre(x'), post and pre RMS or layer norms.
  unjoin    the gradients of that: of x, y and of every vector.

The generator: Philox 4x32 with 7 rounds (Salmon, Moraes, Dror and Shaw, 2011), key = the seed, counter =
(column / 8, row, offset low, offset high).  Its four words are eight halves, low half first; the element of column c looks at
half c % 8 and is dropped where it is below round(65536 p); the others are multiplied by 65536 / (65536 - round(65536 p)).

Sizes come from the workloads in ``workloads.py`` or are generic.  With ``own`` unset the operators are computed by
elementary torch operations in 32 bits; ``exact`` computes them from the definition in 64.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
EPS = 1e-5


# ---------------------------------------------------------------------------
# Which cases
# ---------------------------------------------------------------------------
def _linear(kind, name, M, K, N, mode, ratio, dtype, act, bias, gate, p, residual=False, keep_z=False):
    c = dict(kind=kind, M=M, K=K, N=N, mode=mode, ratio=ratio, dtype=dtype, act=act, bias=bias, gate=gate, p=p)
    if kind == "product":
        c.update(residual=residual, keep_z=keep_z)
    return dict(name=name, **c) if name else c


def _dropout(name, rows, cols, p, dtype="bf16"):
    c = dict(kind="dropout", rows=rows, cols=cols, p=p, dtype=dtype)
    return dict(name=name, **c) if name else c


def _join(kind, name, rows, cols, norm, post, pre, p, bias, gate, scale, dtype="bf16"):
    c = dict(kind=kind, rows=rows, cols=cols, norm=norm, post=post, pre=pre, p=p, bias=bias, gate=gate, scale=scale, dtype=dtype)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # one token of one user: silu(x Wg) * up of a gated MLP, the shard is read once and the rest is latency
        _linear("product", "serve-1-token-gate", 1, 4096, 2752, "n", 0.0, "bf16", "silu", False, True, 0.0),
        # the first product of an MLP in training: bias, GELU, and what its backward pass needs is kept
        _linear("product", "fwd-gpt2-medium-fc1", 8 * 1024, 1024, 1024, "n", 0.0, "bf16", "gelu_tanh", True, False, 0.0, keep_z=True),
        # the headline workload's gate projection with a quarter of its features pruned
        _linear("product", "fwd-llama2-7b-gate", 8192, 4096, 2752, "n", 0.25, "bf16", "silu", False, True, 0.0, keep_z=True),
        # odd extents everywhere, fp32, part of the contraction pruned, dropout and residual
        _linear("product", "fwd-ragged-fp32", 5 * 197, 1001, 771, "k", 0.25, "f32", "none", True, False, 0.1, residual=True),
        # the image model's first projection, pruned: 12608 tokens
        _linear("backward", "bwd-vit-large-fc1", 64 * 197, 1024, 2048, "n", 0.2, "bf16", "gelu", True, False, 0.0),
        # five sequences, odd extents, gated, dropout
        _linear("backward", "bwd-ragged", 5 * 197, 771, 1001, "k", 0.25, "bf16", "silu", True, True, 0.1),
        # one sequence of a narrow model: the launch is what it costs
        _dropout("dropout-small", 197, 1023, 0.1),
        # the residual stream of the headline workload
        _dropout("dropout-8192x4096", 8192, 4096, 0.1),
        # one token: norm after and before a block, a gate per feature
        _join("join", "join-1-token", 1, 4096, "rms", True, True, 0.0, False, True, 1.0),
        # training, image model: bias, dropout, residual and the next layer norm
        _join("join", "join-vit-large", 64 * 197, 1024, "layer", False, True, 0.1, True, True, 1.0),
        # its backward pass over the headline workload's tokens, norms on both sides
        _join("unjoin", "unjoin-8192x4096", 8192, 4096, "rms", True, True, 0.0, False, True, 0.5),
        # fp32 and a width that no vector load fits
        _join("unjoin", "unjoin-ragged-fp32", 5 * 197, 1023, "layer", True, True, 0.1, True, True, 0.7, dtype="f32"),
    ]


def _log(rng, lo, hi, step=1):
    """An integer in [lo, hi], uniform in its logarithm, a multiple of `step`."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return int(min(hi, max(lo, round(v / step) * step)))


def draw(rng):
    kind = rng.choice(["product", "product", "product", "backward", "backward", "dropout", "join", "join", "unjoin", "unjoin"])
    step = rng.choice([1, 8, 64])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    p = 0.0 if rng.random() < 0.4 else round(rng.uniform(0.01, 0.6), 3)
    flag = lambda: rng.random() < 0.5           # noqa: E731
    if kind == "dropout":
        return _dropout(None, _log(rng, 1, 12608), _log(rng, 8, 5120, step), p or 0.1, dtype)
    if kind in ("join", "unjoin"):
        post, pre = rng.choice([(True, True), (False, True), (False, True), (True, False), (False, False)])
        rows, cols = _log(rng, 1, 12608), _log(rng, 8, 5120, step)
        return _join(kind, None, rows, cols, rng.choice(["rms", "layer"]), post, pre, p, flag(), flag(),
                     rng.choice([1.0, 0.5, round(rng.uniform(0.1, 2.0), 3)]), dtype)
    ratio = 0.0 if rng.random() < 0.4 else round(rng.uniform(0.02, 0.6), 3)
    K, N = _log(rng, 64, 5120, step), _log(rng, 64, 5120, step)
    most = (1.0 if dtype == "bf16" else 0.1) * 8192 * 4096 * 2752
    M = max(1, min(_log(rng, 1, 12608), int(most / (K * N * (1 if kind == "product" else 2)))))
    return _linear(kind, None, M, K, N, rng.choice(["n", "k"]), ratio, dtype, rng.choice(ACTS), flag(), flag(), p, flag(), flag())


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _kept(n, ratio):
    return max(1, math.floor((1.0 - ratio) * n + 0.5))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    def activation(rows, cols):         # channels of unlike size, as in trained layers
        return (normal(rows, cols) * torch.exp(0.7 * normal(1, cols))).to(dtype)

    s = dict(case=case)
    # seed and position of the generator
    s["rng"] = torch.tensor([(seed * 0x9E3779B97F4A7C15 + 77) % (1 << 63), (seed * 40503 << 20) % (1 << 62)], dtype=torch.int64, device="cuda")
    if case["kind"] == "dropout":
        s["x"] = activation(case["rows"], case["cols"])
        s["out"] = torch.empty_like(s["x"])
        return s
    if case["kind"] in ("join", "unjoin"):
        rows, cols = case["rows"], case["cols"]
        vec = lambda at, size: (at + size * normal(cols)).to(dtype)         # noqa: E731
        s["y"] = activation(rows, cols)
        s["bias"] = vec(0.0, 0.1) if case["bias"] else None
        s["gate"] = vec(0.5, 0.2) if case["gate"] else None
        for side in ("post", "pre"):
            s[side + "_w"] = vec(1.0, 0.2) if case[side] else None
            s[side + "_b"] = vec(0.0, 0.2) if case[side] and case["norm"] == "layer" else None
        # the residual stream: larger than a block's output, with a mean
        s["x"] = (activation(rows, cols).float() * 2.0 + 0.1).to(dtype)
        if case["kind"] == "join":
            s["x_out"] = torch.empty_like(s["x"])
            s["h"] = torch.empty_like(s["x"]) if case["pre"] else None
            return s
        s["dx_out"] = (0.1 * normal(rows, cols)).to(dtype)
        s["dh"] = (0.1 * normal(rows, cols)).to(dtype) if case["pre"] else None
        s["dx"], s["dy"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
        for v in ("bias", "gate", "post_w", "post_b", "pre_w", "pre_b"):
            s["d" + v] = torch.empty_like(s[v]) if s[v] is not None else None
        if own:
            from paper_2401_11469_amd import zr
            s["ws"] = torch.empty(zr.block_join_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
        return s
    M, K, N, mode = case["M"], case["K"], case["N"], case["mode"]
    n = N if mode == "n" else K
    s["keep"] = torch.randperm(n, generator=gen, device="cuda")[:_kept(n, case["ratio"])].sort()[0].to(torch.int32) if case["ratio"] else None
    s["X"] = activation(M, K)
    # the weight as the layer stores it: its pruned axis is the row axis
    s["W"] = (0.02 * normal(*((N, K) if mode == "n" else (K, N)))).to(dtype)
    s["bias"] = (0.1 * normal(N)).to(dtype) if case["bias"] else None
    s["gate"] = normal(M, N).to(dtype) if case["gate"] else None
    if case["kind"] == "product":
        s["residual"] = activation(M, N) if case["residual"] else None
        s["Y"] = torch.empty((M, N), dtype=dtype, device="cuda")
        s["Z"] = torch.empty_like(s["Y"]) if case["keep_z"] else None
    else:
        s["Z"] = (1.5 * normal(M, N)).to(dtype)
        s["dY"] = (0.1 * normal(M, N)).to(dtype)
        s["dX"], s["dW"] = torch.empty_like(s["X"]), torch.empty_like(s["W"])
        s["dbias"] = torch.empty_like(s["bias"]) if case["bias"] else None
        s["dgate"] = torch.empty_like(s["dY"]) if case["gate"] else None
    if own:             # the scratch buffer that a program allocates once
        from paper_2401_11469_amd import zr
        size = zr.act_workspace_bytes(M, K, N, s["keep"].numel() if case["ratio"] else n, zr.DROP_N if mode == "n" else zr.DROP_K,
                                      dtype, backward=case["kind"] == "backward")
        s["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------
# Plain form: elementary torch operations in 32 bits
# ---------------------------------------------------------------------------
def _factor(rng, rows, cols, p):
    """What dropout multiplies each element by, [rows, cols] in 32 bits."""
    q = min(65535, int(math.floor(p * 65536.0 + 0.5)))
    if q == 0:
        return torch.ones((rows, cols), device=rng.device)
    low = 0xFFFFFFFF
    key0, key1 = rng[0] & low, (rng[0] >> 32) & low
    groups = (cols + 7) // 8
    shape = (rows, groups)
    c0 = torch.arange(groups, device=rng.device).expand(shape)
    c1 = torch.arange(rows, device=rng.device)[:, None].expand(shape)
    c2, c3 = (rng[1] & low).expand(shape), ((rng[1] >> 32) & low).expand(shape)
    for _ in range(7):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57         # (64 bits, wrapped)
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ key0, b & low, ((a >> 32) & low) ^ c3 ^ key1, a & low
        key0, key1 = (key0 + 0x9E3779B9) & low, (key1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], dim=-1)
    halves = torch.stack([words & 0xFFFF, words >> 16], dim=-1).reshape(rows, groups * 8)[:, :cols]
    return (halves >= q).float() * (65536.0 / (65536.0 - q))


def _act(z, act):
    """The activation and its derivative."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        on = (z > 0).float()
        return z * on, on
    if act == "gelu":
        cdf = 0.5 * torch.special.erfc(-z * math.sqrt(0.5))
        return z * cdf, cdf + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "silu":
        t = 1.0 / (1.0 + torch.exp(-z))
        return z * t, t * (1.0 + z * (1.0 - t))
    u = math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)
    t = 1.0 / (1.0 + torch.exp(-2.0 * u))               # (1 + tanh u) / 2
    return z * t, t + z * t * (1.0 - t) * 2.0 * math.sqrt(2.0 / math.pi) * (1.0 + 0.134145 * z * z)


def _spread(kept, n, axis, keep):
    """Kept slices at their places, zeros between them."""
    if keep is None:
        return kept
    shape = list(kept.shape)
    shape[axis] = n
    return torch.zeros(shape, dtype=kept.dtype, device=kept.device).index_copy_(axis, keep.long(), kept)


def _rows(W, keep):
    return W.float() if keep is None else W[keep.long()].float()


def _cols(x, keep):
    return x if keep is None else x[:, keep.long()]


def _plain_product(s):
    c, keep, dt = s["case"], s["keep"], DTYPES[s["case"]["dtype"]]
    X, W = s["X"].float(), _rows(s["W"], keep)
    z = _cols(X, keep) @ W if c["mode"] == "k" else _spread(X @ W.t(), c["N"], 1, keep)
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(z, c["act"])[0]
    if s["gate"] is not None:
        y = y * s["gate"].float()
    y = y * _factor(s["rng"], c["M"], c["N"], c["p"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return (y.to(dt), z.to(dt)) if c["keep_z"] else y.to(dt)


def _plain_backward(s):
    c, keep, dt = s["case"], s["keep"], DTYPES[s["case"]["dtype"]]
    X, W = s["X"].float(), _rows(s["W"], keep)
    a, slope = _act(s["Z"].float(), c["act"])
    t = s["dY"].float() * _factor(s["rng"], c["M"], c["N"], c["p"])
    dz = t * slope
    if s["gate"] is not None:
        dz = dz * s["gate"].float()
    if c["mode"] == "k":
        dX, dW = _spread(dz @ W.t(), c["K"], 1, keep), _spread(_cols(X, keep).t() @ dz, c["K"], 0, keep)
    else:
        kept = _cols(dz, keep)
        dX, dW = kept @ W, _spread(kept.t() @ X, c["N"], 0, keep)
    out = [dX, dW]
    if s["bias"] is not None:
        out.append(dz.sum(dim=0, dtype=torch.float64))
    if s["gate"] is not None:
        out.append(t * a)
    return tuple(o.to(dt) for o in out)


def _norm(v, norm):
    """(the normalised rows, one over their deviation)"""
    if norm == "layer":
        v = v - v.mean(dim=1, keepdim=True)
    r = 1.0 / torch.sqrt((v * v).mean(dim=1, keepdim=True) + EPS)
    return v * r, r


def _norm_back(g, hat, r, norm):
    d = g - hat * (g * hat).mean(dim=1, keepdim=True)
    if norm == "layer":
        d = d - g.mean(dim=1, keepdim=True)
    return d * r


def _f(v, other):
    return other if v is None else v.float()


def _plain_join(s):
    c, dt = s["case"], DTYPES[s["case"]["dtype"]]
    n = (s["y"].float() + _f(s["bias"], 0.0)) * _factor(s["rng"], c["rows"], c["cols"], c["p"])
    if c["post"]:
        n = _norm(n, c["norm"])[0] * s["post_w"].float() + _f(s["post_b"], 0.0)
    x = s["x"].float() + c["scale"] * _f(s["gate"], 1.0) * n
    if not c["pre"]:
        return x.to(dt)
    h = _norm(x, c["norm"])[0] * s["pre_w"].float() + _f(s["pre_b"], 0.0)
    return x.to(dt), h.to(dt)


def _plain_unjoin(s):
    """`x` of the state is the residual stream behind the block here."""
    c, dt = s["case"], DTYPES[s["case"]["dtype"]]
    out = {}
    dx = s["dx_out"].float()
    if c["pre"]:
        dh = s["dh"].float()
        hat, r = _norm(s["x"].float(), c["norm"])
        dx = dx + _norm_back(dh * s["pre_w"].float(), hat, r, c["norm"])
        out["pre_w"] = (dh * hat).sum(dim=0, dtype=torch.float64)
        out["pre_b"] = dh.sum(dim=0, dtype=torch.float64)
    f = _factor(s["rng"], c["rows"], c["cols"], c["p"])
    n = t = (s["y"].float() + _f(s["bias"], 0.0)) * f
    if c["post"]:
        hat, r = _norm(t, c["norm"])
        n = hat * s["post_w"].float() + _f(s["post_b"], 0.0)
    out["gate"] = (c["scale"] * dx * n).sum(dim=0, dtype=torch.float64)
    dn = c["scale"] * dx * _f(s["gate"], 1.0)
    dt_ = dn
    if c["post"]:
        out["post_w"] = (dn * hat).sum(dim=0, dtype=torch.float64)
        out["post_b"] = dn.sum(dim=0, dtype=torch.float64)
        dt_ = _norm_back(dn * s["post_w"].float(), hat, r, c["norm"])
    dy = dt_ * f
    out["bias"] = dy.sum(dim=0, dtype=torch.float64)
    vectors = [out[v] for v in ("bias", "gate", "post_w", "post_b", "pre_w", "pre_b") if s[v] is not None]
    return tuple(o.to(dt) for o in [dx, dy, *vectors])


def _plain(s):
    c = s["case"]
    if c["kind"] == "dropout":
        return (s["x"].float() * _factor(s["rng"], c["rows"], c["cols"], c["p"])).to(DTYPES[c["dtype"]])
    return {"product": _plain_product, "backward": _plain_backward, "join": _plain_join, "unjoin": _plain_unjoin}[c["kind"]](s)


# ---------------------------------------------------------------------------
# The framework's calls
# ---------------------------------------------------------------------------
def _own(s):
    from paper_2401_11469_amd import zr
    c = s["case"]
    if c["kind"] == "dropout":
        return zr.dropout(s["x"], c["p"], s["rng"], out=s["out"])
    if c["kind"] in ("join", "unjoin"):
        how = dict(norm=zr.NORM_RMS if c["norm"] == "rms" else zr.NORM_LAYER, post=c["post"], pre=c["pre"], eps=EPS, p=c["p"], rng=s["rng"],
                   scale=c["scale"], bias=s["bias"], gate=s["gate"], post_w=s["post_w"], post_b=s["post_b"], pre_w=s["pre_w"])
        if c["kind"] == "join":
            out = zr.block_join_fwd(s["y"], s["x"], **how, pre_b=s["pre_b"], x_out=s["x_out"], h=s["h"])
            return out if c["pre"] else out[0]
        zr.block_join_bwd(s["dx_out"], s["dh"], s["x"] if c["pre"] else None, s["y"], **how, dx=s["dx"], dy=s["dy"], dbias=s["dbias"],
                          dgate=s["dgate"], dpost_w=s["dpost_w"], dpost_b=s["dpost_b"], dpre_w=s["dpre_w"], dpre_b=s["dpre_b"],
                          workspace=s["ws"])
        return tuple(s[o] for o in ("dx", "dy", "dbias", "dgate", "dpost_w", "dpost_b", "dpre_w", "dpre_b") if s[o] is not None)
    how = dict(mode=zr.DROP_N if c["mode"] == "n" else zr.DROP_K, w_layout=zr.W_NK if c["mode"] == "n" else zr.W_KN,
               act={"none": zr.ACT_NONE, "relu": zr.ACT_RELU, "gelu": zr.ACT_GELU, "gelu_tanh": zr.ACT_GELU_TANH, "silu": zr.ACT_SILU}[c["act"]],
               gate=s["gate"], p=c["p"], rng=s["rng"], workspace=s["ws"])
    if c["kind"] == "product":
        zr.resized_linear_act_fwd(s["X"], s["W"], s["keep"], bias=s["bias"], residual=s["residual"], Y=s["Y"], Z=s["Z"], **how)
        return (s["Y"], s["Z"]) if c["keep_z"] else s["Y"]
    zr.resized_linear_act_bwd(s["X"], s["W"], s["dY"], s["keep"], Z=s["Z"], dX=s["dX"], dW=s["dW"], dbias=s["dbias"], dgate=s["dgate"], **how)
    return tuple(s[o] for o in ("dX", "dW", "dbias", "dgate") if s[o] is not None)


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# What a pass cannot do without, and what it gives in 64 bits
# ---------------------------------------------------------------------------
def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": 2.0 * n * es, "flops": 1.0 * n}
    if case["kind"] in ("join", "unjoin"):
        n, vectors = case["rows"] * case["cols"], case["cols"] * es * (case["bias"] + case["gate"] + (case["post"] + case["pre"]) * (1 + (case["norm"] == "layer")))
        # y, x -> x', h;   dx', dh, x' and y (where something depends on it) -> dx, dy
        tensors = 3 + case["pre"] if case["kind"] == "join" else 3 + 2 * case["pre"] + (case["post"] or case["gate"])
        return {"bytes": 1.0 * n * es * tensors + vectors * (1 if case["kind"] == "join" else 2),
                "flops": 1.0 * n * (4 + 8 * (case["post"] + case["pre"])) * (1 if case["kind"] == "join" else 2)}
    M, K, N = case["M"], case["K"], case["N"]
    n = _kept(N if case["mode"] == "n" else K, case["ratio"])
    k, j = (K, n) if case["mode"] == "n" else (n, N)        # the kept extents of W
    if case["kind"] == "product":
        planes = 1 + case["gate"] + case["residual"] + case["keep_z"]
        return {"bytes": es * (1.0 * M * k + k * j + M * N * planes + N * case["bias"]), "flops": 2.0 * M * k * j}
    planes = 1 + (case["act"] != "none" or case["gate"]) + 2 * case["gate"]
    return {"bytes": es * (1.0 * M * N * planes + M * k + k * j + M * K + K * N + N * case["bias"]), "flops": 4.0 * M * k * j}


def _exact_factor(rng, rows, cols, p):
    q = min(65535, int(math.floor(p * 65536.0 + 0.5)))
    if q == 0:
        return 1.0
    seed, offset = (int(v) & (2 ** 64 - 1) for v in rng.cpu().tolist())
    u = np.uint64
    low, half = u(0xFFFFFFFF), u(32)
    groups = -(-cols // 8)
    x = [np.broadcast_to(v, (rows, groups)) for v in (np.arange(groups, dtype=u)[None, :], np.arange(rows, dtype=u)[:, None],
                                                      np.array(offset, dtype=u) & low, np.array(offset, dtype=u) >> half)]
    for i in range(7):
        k0 = u((seed + i * 0x9E3779B9) % 2 ** 32)
        k1 = u(((seed >> 32) + i * 0xBB67AE85) % 2 ** 32)
        first, second = x[0] * u(0xD2511F53), x[2] * u(0xCD9E8D57)
        x = [(second >> half) ^ x[1] ^ k0, second & low, (first >> half) ^ x[3] ^ k1, first & low]
    kept = np.empty((rows, groups, 8), dtype=bool)
    for w in range(4):
        kept[:, :, 2 * w] = (x[w] & u(0xFFFF)) >= u(q)
        kept[:, :, 2 * w + 1] = (x[w] >> u(16)) >= u(q)
    return torch.from_numpy(kept.reshape(rows, -1)[:, :cols].copy()).to(rng.device).double() * (65536.0 / (65536 - q))


def _exact_act(z, act):
    one = torch.ones_like(z)
    if act == "relu":
        return torch.where(z > 0, z, 0 * one), torch.where(z > 0, one, 0 * one)
    if act == "gelu":
        tail = torch.special.erfc(-z / 2 ** 0.5) / 2
        return z * tail, tail + z * torch.exp(-z ** 2 / 2) / (2 * math.pi) ** 0.5
    if act == "gelu_tanh":
        b = (2 / math.pi) ** 0.5
        s = torch.sigmoid(2 * b * (z + 0.044715 * z ** 3))          # (1 + tanh u) / 2
        return z * s, s + z * 2 * s * torch.sigmoid(-2 * b * (z + 0.044715 * z ** 3)) * b * (1 + 3 * 0.044715 * z ** 2)
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * torch.sigmoid(-z)
    return z, one


def _exact_linear(s):
    c, mode = s["case"], s["case"]["mode"]
    keep = s["keep"].long() if s["keep"] is not None else torch.arange(c["N"] if mode == "n" else c["K"], device="cuda")
    X, w = s["X"].double(), s["W"].double()[keep]
    f = _exact_factor(s["rng"], c["M"], c["N"], c["p"])
    gate = 1.0 if s["gate"] is None else s["gate"].double()
    if c["kind"] == "product":
        if mode == "k":
            z = X[:, keep] @ w
        else:
            z = torch.zeros((c["M"], c["N"]), dtype=torch.float64, device="cuda")
            z[:, keep] = X @ w.t()
        if s["bias"] is not None:
            z = z + s["bias"].double()[None, :]
        y = _exact_act(z, c["act"])[0] * gate * f
        if s["residual"] is not None:
            y = y + s["residual"].double()
        return (y, z) if c["keep_z"] else y
    a, slope = _exact_act(s["Z"].double(), c["act"])
    t = s["dY"].double() * f
    dz = t * gate * slope
    dW = torch.zeros(s["W"].shape, dtype=torch.float64, device="cuda")
    if mode == "k":
        dX = torch.zeros(X.shape, dtype=torch.float64, device="cuda")
        dX[:, keep] = dz @ w.t()
        dW[keep] = X[:, keep].t() @ dz
    else:
        dX = dz[:, keep] @ w
        dW[keep] = dz[:, keep].t() @ X
    out = [dX, dW]
    if s["bias"] is not None:
        out.append(dz.sum(dim=0))
    if s["gate"] is not None:
        out.append(t * a)
    return tuple(out)


def _exact_hat(v, norm):
    if norm == "layer":
        v = v - v.sum(dim=1, keepdim=True) / v.shape[1]
    dev = torch.sqrt((v ** 2).sum(dim=1, keepdim=True) / v.shape[1] + EPS)
    return v / dev, dev


def _exact_hat_back(g, hat, dev, norm):
    n = g.shape[1]
    along = (g * hat).sum(dim=1, keepdim=True) / n
    level = g.sum(dim=1, keepdim=True) / n if norm == "layer" else 0.0
    return (g - level - hat * along) / dev


def _exact_join(s):
    c = s["case"]
    d = {v: None if s[v] is None else s[v].double() for v in ("y", "x", "bias", "gate", "post_w", "post_b", "pre_w", "pre_b")}
    f = _exact_factor(s["rng"], c["rows"], c["cols"], c["p"])
    gate = (1.0 if d["gate"] is None else d["gate"]) * c["scale"]
    t = (d["y"] if d["bias"] is None else d["y"] + d["bias"]) * f
    n = t
    if c["post"]:
        hat, dev = _exact_hat(t, c["norm"])
        n = hat * d["post_w"] if d["post_b"] is None else hat * d["post_w"] + d["post_b"]
    if c["kind"] == "join":
        x = d["x"] + gate * n
        if not c["pre"]:
            return x
        h = _exact_hat(x, c["norm"])[0] * d["pre_w"]
        return x, (h if d["pre_b"] is None else h + d["pre_b"])
    dx = s["dx_out"].double()
    sums = {}
    if c["pre"]:
        dh = s["dh"].double()
        top, top_dev = _exact_hat(d["x"], c["norm"])
        dx = dx + _exact_hat_back(dh * d["pre_w"], top, top_dev, c["norm"])
        sums["pre_w"], sums["pre_b"] = dh * top, dh
    sums["gate"] = dx * n * c["scale"]
    dn = dx * gate
    if c["post"]:
        sums["post_w"], sums["post_b"] = dn * hat, dn
        dn = _exact_hat_back(dn * d["post_w"], hat, dev, c["norm"])
    dy = dn * f
    sums["bias"] = dy
    return tuple([dx, dy] + [sums[v].sum(dim=0) for v in ("bias", "gate", "post_w", "post_b", "pre_w", "pre_b") if d[v] is not None])


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "dropout":
        return s["x"].double() * _exact_factor(s["rng"], case["rows"], case["cols"], case["p"])
    return _exact_linear(s) if case["kind"] in ("product", "backward") else _exact_join(s)
