"""The low-bit operators of the resized linear layer, as cases that can be timed and checked.

Values are held in blocks of 32 along the axis that a product sums over: one power of two per block and 8 or 4 bits per
value (E4M3, E2M1 or an 8-bit integer in 64ths).  A case is one of these kinds of work:

  store     an activation (its kept columns) or a weight shard (its kept rows) is put into blocks and read back: the
            activation checkpoint of a layer, and what a weight loader does.  The values come back in the tensor's type.
  product   Y from an activation that arrives in the tensor's type and is put into blocks on the way, and a weight shard that
            was put into blocks once; whole, or the kept features / the kept part of the contraction alone.
  backward  dX and dW of the resized layer from the checkpoint of its input.
  step      a training step of one projection: the weight's kept rows and the input's kept columns into blocks, the product,
            and the backward products from the same blocks.

Sizes come from the workloads in ``workloads.py`` or are generic.  With ``own`` unset the operators are computed by
elementary torch operations in 32 bits; ``exact`` computes them from the definition in 64.
"""
from __future__ import annotations

import math

import torch

own = False

# format: the largest value, the power of two of its binade, the smallest binade with a full mantissa, mantissa bits, bits held
FORMATS = {"e4m3": (448.0, 8, -6, 3, 8), "e2m1": (6.0, 2, 0, 1, 4), "int8": (127.0 / 64.0, 0, 0, 6, 8)}
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------
# Which cases
# ---------------------------------------------------------------------------
def _store(name, rows, cols, ratio, fmt, dtype="bf16", axis=1):
    c = dict(kind="store", rows=rows, cols=cols, ratio=ratio, fmt=fmt, dtype=dtype, axis=axis)
    return dict(name=name, **c) if name else c


def _product(name, M, K, N, x_fmt, w_fmt, mode="n", ratio=0.0, dtype="bf16", policy="zero"):
    c = dict(kind="product", M=M, K=K, N=N, x_fmt=x_fmt, w_fmt=w_fmt, mode=mode, ratio=ratio, dtype=dtype, policy=policy)
    return dict(name=name, **c) if name else c


def _backward(name, M, K, N, fmt, mode, ratio, dtype="bf16", policy="zero"):
    c = dict(kind="backward", M=M, K=K, N=N, x_fmt=fmt, mode=mode, ratio=ratio, dtype=dtype, policy=policy)
    return dict(name=name, **c) if name else c


def _step(name, M, K, N, x_fmt, w_fmt, ratio, dtype="bf16"):
    c = dict(kind="step", M=M, K=K, N=N, x_fmt=x_fmt, w_fmt=w_fmt, mode="k", ratio=ratio, dtype=dtype, policy="zero")
    return dict(name=name, **c) if name else c


def listed():
    return [
        # the smallest checkpoint: one sequence's rows of a narrow row-parallel shard, launches are what it costs
        _store("store-gpt2-out-small", 197, 256, 0.25, "int8"),
        # the checkpoint of a row-parallel input of the headline workload, a quarter of its columns pruned
        _store("store-llama2-7b-down", 8192, 2752, 0.25, "e4m3"),
        # fp32 training with rows that no vector load fits, nothing pruned
        _store("store-fp32-ragged", 8 * 197, 2047, 0.0, "int8", dtype="f32"),
        # a weight loader: a row-parallel shard stored [in x out] into 4 bits along its inputs
        _store("store-weight-4bit", 5120, 1728, 0.0, "e2m1", axis=0),
        # one token of one user: a 4-bit shard has to be read once, the rest is latency
        _product("serve-1-token", 1, 4096, 2752, "e4m3", "e2m1"),
        # a decoding batch, everything in 4 bits
        _product("serve-48-tokens", 48, 5120, 1728, "e2m1", "e2m1"),
        # a column-parallel forward over the headline workload's tokens, a quarter of the features pruned
        _product("prefill-llama2-7b-gate", 8192, 4096, 2752, "e2m1", "e2m1", ratio=0.25),
        # five images, odd extents everywhere, fp32 results, part of the contraction pruned
        _product("product-ragged-fp32", 5 * 197, 1001, 771, "e4m3", "e2m1", mode="k", ratio=0.25, dtype="f32"),
        # the backward products of the headline workload's row-parallel projection
        _backward("backward-llama2-7b-down", 8192, 2752, 4096, "e4m3", "k", 0.25),
        # the image model's column-parallel projection: odd token count, integer checkpoint, the previous values imputed
        _backward("backward-vit-large-fc1", 64 * 197, 1024, 2048, "int8", "n", 0.2, policy="same"),
        # the tiny fp32 linear
        _backward("backward-tiny-fp32", 256, 512, 256, "int8", "n", 0.25, dtype="f32"),
        # a whole training step of one projection, 8-bit operands
        _step("step-llama2-7b-down", 8192, 2752, 4096, "e4m3", "e4m3", 0.25),
    ]


def _log(rng, lo, hi, step=1):
    """An integer in [lo, hi], uniform in its logarithm, a multiple of `step`."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return int(min(hi, max(lo, round(v / step) * step)))


def draw(rng):
    kind = rng.choice(["store", "store", "product", "product", "product", "backward", "backward", "step"])
    ratio = 0.0 if rng.random() < 0.2 else round(rng.uniform(0.02, 0.6), 3)
    step = rng.choice([1, 8, 64])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "store":
        rows, cols = _log(rng, 1, 16384), _log(rng, 32, 12288, step)
        return _store(None, rows, cols, ratio, rng.choice(["e4m3", "e2m1", "int8"]), dtype, axis=rng.choice([1, 1, 0]))
    K, N = _log(rng, 64, 5120, step), _log(rng, 64, 5120, step)
    most = (2.0 if dtype == "bf16" else 0.2) * 8192 * 2064 * 4096
    policy = rng.choice(["zero", "zero", "same", "average"])
    if kind == "product":
        M = max(1, min(_log(rng, 1, 16384), int(most / (K * N))))
        x_fmt, w_fmt = rng.choice([("e4m3", "e2m1"), ("e2m1", "e2m1"), ("e4m3", "e4m3")])
        return _product(None, M, K, N, x_fmt, w_fmt, rng.choice(["n", "k"]), ratio, dtype, policy)
    M = max(1, min(_log(rng, 16, 16384), int(most / (2 * K * N))))
    if kind == "backward":
        return _backward(None, M, K, N, rng.choice(["e4m3", "int8"]), rng.choice(["n", "k"]), ratio, dtype, policy)
    return _step(None, M, K, N, "e4m3", rng.choice(["e4m3", "e2m1"]), ratio, dtype)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _kept(n, ratio):
    return max(1, math.floor((1.0 - ratio) * n + 0.5))


def _row_bytes(n, fmt):
    """Bytes of a row's values: whole groups of 128 of them."""
    return (n + 127) // 128 * 128 * FORMATS[fmt][4] // 8


def _scale_bytes(n):
    """Bytes of a row's powers of two: groups of 16 blocks."""
    return (n + 511) // 512 * 16


def _buffers(rows, n, fmt):
    return (torch.empty((rows, _row_bytes(n, fmt)), dtype=torch.uint8, device="cuda"),
            torch.empty((rows, _scale_bytes(n)), dtype=torch.uint8, device="cuda"))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    def activation(rows, cols):         # channels of unlike size, as in trained layers
        return (normal(rows, cols) * torch.exp(0.7 * normal(1, cols))).to(dtype)

    def kept_list(n):
        return torch.randperm(n, generator=gen, device="cuda")[:_kept(n, case["ratio"])].sort()[0].to(torch.int32)

    s = dict(case=case)
    if case["kind"] == "store":
        rows, cols, axis = case["rows"], case["cols"], case["axis"]
        s["src"] = activation(rows, cols) if axis == 1 else (0.02 * normal(rows, cols)).to(dtype)
        s["keep"] = kept_list(cols if axis == 1 else rows) if case["ratio"] else None
        n = s["keep"].numel() if case["ratio"] else (cols if axis == 1 else rows)
        s["n"] = n
        s["mx"] = _buffers(rows if axis == 1 else cols, n, case["fmt"])
        s["out"] = torch.empty((rows if axis == 1 else cols, n), dtype=dtype, device="cuda")
        return s
    M, K, N, mode = case["M"], case["K"], case["N"], case["mode"]
    s["keep"] = kept_list(N if mode == "n" else K)
    n_keep = s["keep"].numel()
    s["nc"] = n_keep if mode == "k" else K                  # the length of the forward contraction
    wide = lambda t: t[:, s["keep"].long()].contiguous() if mode == "k" else t  # noqa: E731
    X = activation(M, K)
    if case["kind"] in ("product", "step"):
        s["X"] = X
        s["Y"] = torch.empty((M, N), dtype=dtype, device="cuda")
        # a server keeps no copy of a few tokens' input; a training step does
        s["x_mx"] = _buffers(M, s["nc"], case["x_fmt"]) if M > 16 or case["kind"] == "step" else None
        s["prev_Y"] = normal(M, N).to(dtype) if case["policy"] == "same" else None
    if case["kind"] == "product":
        s["w_mx"] = _pack(wide((0.02 * normal(N, K)).to(dtype)), case["w_fmt"])
        return s
    # the weight as the layer stores it: its pruned axis is the row axis
    s["W"] = (0.02 * normal(*((N, K) if mode == "n" else (K, N)))).to(dtype)
    s["dY"] = (0.1 * normal(M, N)).to(dtype)
    s["dX"] = torch.empty((M, K), dtype=dtype, device="cuda")
    s["dW"] = torch.empty_like(s["W"])
    same = case["policy"] == "same"
    s["prev_dX"] = normal(M, K).to(dtype) if same else None
    s["prev_dW"] = normal(*s["W"].shape).to(dtype) if same else None
    if case["kind"] == "backward":
        s["x_mx"] = _pack(wide(X), case["x_fmt"])
    else:
        s["w_mx"] = _buffers(N, n_keep, case["w_fmt"])
    if own:             # the scratch buffer that a training program allocates once
        from paper_2401_11469_amd import zr
        size = zr.mx_bwd_workspace_bytes(M, K, N, n_keep, zr.DROP_N if mode == "n" else zr.DROP_K, dtype)
        s["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------
# Plain form: elementary torch operations in 32 bits
# ---------------------------------------------------------------------------
def _powers(exponents):
    """2^e in 32 bits for e in [-127, 127], from the exponent field alone."""
    e = exponents.to(torch.int32)
    return torch.where(e > -127, (e + 127) << 23, torch.full_like(e, 1 << 22)).view(torch.float32)


def _in_blocks(x, fmt):
    """x [rows, n] -> (elements [rows, blocks, 32] on the format's grid, exponents [rows, blocks])."""
    top, emax, emin, mant, _ = FORMATS[fmt]
    x = x.float()
    x = torch.nn.functional.pad(x, (0, -x.shape[1] % 32)).view(x.shape[0], -1, 32)
    a = x.abs().amax(dim=-1)
    m, e = torch.frexp(a)                                   # a = m 2^e, 1/2 <= m < 1
    e = e - 1 - emax + (2.0 * m > top / 2.0 ** emax).to(e.dtype)
    e = torch.where(a > 0, e, torch.full_like(e, -127)).clamp(-127, 127)
    y = x * _powers(-(e // 2))[..., None] * _powers(-(e - e // 2))[..., None]
    binade = torch.frexp(y)[1] - 1
    inv = _powers(mant - binade.clamp(min=emin))
    return torch.round(y * inv) / inv, e


def _values(elements, exponents, n):
    """What the blocks stand for, [rows, n] in 32 bits."""
    e = exponents
    v = elements * _powers(e // 2)[..., None] * _powers(e - e // 2)[..., None]
    return v.reshape(v.shape[0], -1)[:, :n]


def _pack(x, fmt):
    """The stored form of x [rows, n]: values (low nibble first) and powers of two, block b of 16 at byte 4 (b % 4) + b / 4."""
    rows, n = x.shape
    el, e = _in_blocks(x, fmt)
    el = el.reshape(rows, -1)
    el = torch.nn.functional.pad(el, (0, -el.shape[1] % 128))
    if fmt == "int8":
        q = (el * 64.0).to(torch.int8).view(torch.uint8)
    elif fmt == "e4m3":
        q = el.to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=x.device)
        code = torch.searchsorted(grid, el.abs().contiguous()).to(torch.uint8) | ((el < 0).to(torch.uint8) << 3)
        q = code[:, 0::2] | (code[:, 1::2] << 4)
    code = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -e.shape[1] % 16))
    scales = code.view(rows, -1, 4, 4).transpose(2, 3).reshape(rows, -1)
    return q.contiguous(), scales.contiguous()


def _unpack(mx, n, fmt):
    """What the stored form stands for, [rows, n] in 32 bits."""
    q, scales = mx
    rows = q.shape[0]
    e = scales.view(rows, -1, 4, 4).transpose(2, 3).reshape(rows, -1).to(torch.int32) - 127
    if fmt == "int8":
        el = q.view(torch.int8).float() / 64.0
    elif fmt == "e4m3":
        c = torch.arange(256, device=q.device)
        b, m = (c >> 3) & 15, (c & 7).float()
        t = torch.where(b > 0, (8.0 + m) * 2.0 ** (b.float() - 10.0), m * 2.0 ** -9)
        el = torch.where(c > 127, -t, t)[q.long()]
    else:
        t = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=q.device)
        t = torch.cat([t, -t])
        el = t[torch.stack([q & 15, q >> 4], dim=-1).long()].reshape(rows, -1)
    blocks = (n + 31) // 32
    return _values(el[:, :blocks * 32].reshape(rows, blocks, 32), e[:, :blocks], n)


def _fill(kept, n, axis, keep, policy, prev, dtype):
    """A result in its full shape: the kept slices at their places, the others imputed."""
    kept = kept.to(dtype)
    if keep.numel() == n:
        return kept
    shape = list(kept.shape)
    shape[axis] = n
    if policy == "same":
        out = prev.clone()
    elif policy == "average":
        out = kept.float().mean(dim=axis, keepdim=True).to(dtype).expand(shape).clone()
    else:
        out = torch.zeros(shape, dtype=dtype, device=kept.device)
    out.index_copy_(axis, keep.long(), kept)
    return out


def _plain_store(s):
    c = s["case"]
    x = s["src"] if c["axis"] == 1 else s["src"].t()
    if s["keep"] is not None:
        x = x[:, s["keep"].long()]
    el, e = _in_blocks(x, c["fmt"])
    return _values(el, e, x.shape[1]).to(DTYPES[c["dtype"]])


def _plain_fwd(s, xv, wv):
    c = s["case"]
    if c["mode"] == "k":
        return (xv @ wv.t()).to(DTYPES[c["dtype"]])
    return _fill(xv @ wv[s["keep"].long()].t(), c["N"], 1, s["keep"], c["policy"], s["prev_Y"], DTYPES[c["dtype"]])


def _plain_bwd(s, xv):
    """W is [K, N] and pruned along K, or [N, K] and pruned along N: rows either way."""
    c, keep, dt = s["case"], s["keep"], DTYPES[s["case"]["dtype"]]
    W, dY = s["W"][keep.long()].float(), s["dY"].float()
    if c["mode"] == "k":
        return (_fill(dY @ W.t(), c["K"], 1, keep, c["policy"], s["prev_dX"], dt),
                _fill(xv.t() @ dY, c["K"], 0, keep, c["policy"], s["prev_dW"], dt))
    dY = dY[:, keep.long()]
    return (dY @ W).to(dt), _fill(dY.t() @ xv, c["N"], 0, keep, c["policy"], s["prev_dW"], dt)


def _plain(s):
    c = s["case"]
    if c["kind"] == "store":
        return _plain_store(s)
    if c["kind"] == "backward":
        return _plain_bwd(s, _unpack(s["x_mx"], s["nc"], c["x_fmt"]))
    X = s["X"][:, s["keep"].long()] if c["mode"] == "k" else s["X"]
    xv = _values(*_in_blocks(X, c["x_fmt"]), s["nc"])
    if c["kind"] == "product":
        return _plain_fwd(s, xv, _unpack(s["w_mx"], s["nc"], c["w_fmt"]))
    wv = _values(*_in_blocks(s["W"][s["keep"].long()].t(), c["w_fmt"]), s["nc"])
    return (_plain_fwd(s, xv, wv), *_plain_bwd(s, xv))


# ---------------------------------------------------------------------------
# The framework's calls
# ---------------------------------------------------------------------------
def _own(s):
    from paper_2401_11469_amd import zr
    c = s["case"]
    fmt = {"e4m3": zr.MX_E4M3, "e2m1": zr.MX_E2M1, "int8": zr.MX_INT8}
    if c["kind"] == "store":
        mx = zr.MX(*s["mx"], s["n"], fmt[c["fmt"]])
        zr.mx_quantize(s["src"], mx.fmt, axis=c["axis"], keep_idx=s["keep"], out=mx)
        return zr.mx_dequantize(mx, out=s["out"])
    mode = zr.DROP_N if c["mode"] == "n" else zr.DROP_K
    layout = zr.W_NK if c["mode"] == "n" else zr.W_KN
    policy = {"zero": zr.ZERO, "same": zr.SAME, "average": zr.AVERAGE}[c["policy"]]
    x_mx = zr.MX(*s["x_mx"], s["nc"], fmt[c["x_fmt"]]) if s["x_mx"] is not None else None
    out = []
    if c["kind"] != "backward":
        w_mx = zr.MX(*s["w_mx"], s["nc"], fmt[c["w_fmt"]])
        if c["kind"] == "step":
            zr.mx_quantize(s["W"], w_mx.fmt, axis=0, keep_idx=s["keep"], out=w_mx)
        out.append(zr.mx_linear_fwd(s["X"], w_mx, s["keep"], mode, policy, prev_Y=s["prev_Y"], Y=s["Y"],
                                    x_fmt=fmt[c["x_fmt"]], x_mx=x_mx))
    if c["kind"] != "product":
        out += zr.resized_linear_bwd_mx(x_mx, s["W"], s["dY"], s["keep"], mode, policy, prev_dX=s["prev_dX"],
                                        prev_dW=s["prev_dW"], dX=s["dX"], dW=s["dW"], workspace=s["ws"], w_layout=layout)
    return out[0] if len(out) == 1 else tuple(out)


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# What a pass cannot do without, and what it gives in 64 bits
# ---------------------------------------------------------------------------
def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    held = lambda fmt: FORMATS[fmt][4] / 8 + 1 / 32         # noqa: E731  bytes of a value in blocks
    if case["kind"] == "store":
        rows, cols = case["rows"], case["cols"]
        n = _kept(cols if case["axis"] == 1 else rows, case["ratio"])
        kept = rows * n if case["axis"] == 1 else n * cols
        return {"bytes": kept * (2 * es + 2 * held(case["fmt"])), "flops": 4.0 * kept}
    M, K, N = case["M"], case["K"], case["N"]
    n = _kept(N if case["mode"] == "n" else K, case["ratio"])
    k, j = (K, n) if case["mode"] == "n" else (n, N)        # the kept extents of W
    one = 2.0 * M * k * j
    fwd = {"bytes": M * k * es + M * N * es, "flops": one}
    bwd = {"bytes": es * (M * N + k * j + M * K + K * N) + (0 if case["kind"] == "step" else M * k * held(case["x_fmt"])),
           "flops": 2 * one}
    if case["kind"] == "product":
        return {"bytes": fwd["bytes"] + k * j * held(case["w_fmt"]), "flops": one}
    if case["kind"] == "backward":
        return bwd
    return {"bytes": fwd["bytes"] + bwd["bytes"] + 2 * M * k * held(case["x_fmt"]) + 2 * k * j * held(case["w_fmt"]), "flops": 3 * one}


def _grid(fmt):
    """The non-negative values of a format, ascending."""
    top, _, emin, mant, _ = FORMATS[fmt]
    if fmt == "int8":
        v = [i / 64.0 for i in range(128)]
    else:
        v = [i * 2.0 ** (emin - mant) for i in range(2 ** mant)]
        e = emin
        while v[-1] < top:
            v += [(1.0 + i / 2 ** mant) * 2.0 ** e for i in range(2 ** mant)]
            e += 1
        v = [x for x in v if x <= top]
    return torch.tensor(v, dtype=torch.float64, device="cuda")


def _exact_values(x, fmt):
    """x [rows, n] as its blocks hold it, in 64 bits: the nearest grid value, of two equally near ones the even one."""
    rows, n = x.shape
    out = torch.zeros((rows, (n + 31) // 32 * 32), dtype=torch.float64, device=x.device)
    out[:, :n] = x.double()
    out = out.view(rows, -1, 32)
    a = out.abs().max(dim=2, keepdim=True)[0]
    e = torch.ceil(torch.log2(torch.where(a > 0, a, torch.ones_like(a)) / FORMATS[fmt][0])).clamp(-127, 127)
    y = out / torch.exp2(e)
    grid = _grid(fmt)
    mids = (grid[1:] + grid[:-1]) / 2
    i = torch.searchsorted(mids, y.abs().contiguous())
    tie = (i < mids.numel()) & (mids[i.clamp(max=mids.numel() - 1)] == y.abs())
    i = i + (tie & (i % 2 == 1)).to(i.dtype)
    return (torch.sign(y) * grid[i] * torch.exp2(e)).reshape(rows, -1)[:, :n]


def _exact_spread(kept, n, axis, keep, policy, prev):
    if policy == "same":
        full = prev.double()
    else:
        shape = [n if d == axis else kept.shape[d] for d in range(2)]
        full = torch.zeros(shape, dtype=torch.float64, device=kept.device)
        if policy == "average":
            full = full + kept.mean(dim=axis, keepdim=True)
    if axis == 0:
        full[keep.long()] = kept
    else:
        full[:, keep.long()] = kept
    return full


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "store":
        x = s["src"] if case["axis"] == 1 else s["src"].t().contiguous()
        return _exact_values(x if s["keep"] is None else x[:, s["keep"].long()], case["fmt"])
    keep, mode, policy = s["keep"].long(), case["mode"], case["policy"]
    if case["kind"] == "backward":
        # what the checkpoint holds is an input here; it is read as stored
        x = _exact_held(s["x_mx"], s["nc"], case["x_fmt"])
    else:
        x = _exact_values(s["X"][:, keep] if mode == "k" else s["X"], case["x_fmt"])
    out = []
    if case["kind"] != "backward":
        w = (_exact_held(s["w_mx"], s["nc"], case["w_fmt"]) if case["kind"] == "product"
             else _exact_values(s["W"][keep].t().contiguous(), case["w_fmt"]))
        out.append(x @ w.t() if mode == "k" else _exact_spread(x @ w[keep].t(), case["N"], 1, keep, policy, s["prev_Y"]))
    if case["kind"] != "product":
        w, dy = s["W"][keep].double(), s["dY"].double()
        if mode == "k":
            out.append(_exact_spread(dy @ w.t(), case["K"], 1, keep, policy, s["prev_dX"]))
            out.append(_exact_spread(x.t() @ dy, case["K"], 0, keep, policy, s["prev_dW"]))
        else:
            dy = dy[:, keep]
            out.append(dy @ w)
            out.append(_exact_spread(dy.t() @ x, case["N"], 0, keep, policy, s["prev_dW"]))
    return out[0] if len(out) == 1 else tuple(out)


def _exact_held(mx, n, fmt):
    """The stored form read back in 64 bits, byte by byte from the format's definition."""
    q, scales = (t.long() for t in mx)
    i = torch.arange(n, device=q.device)
    b = i // 32
    e = scales[:, b // 16 * 16 + 4 * (b % 4) + b % 16 // 4] - 127
    if fmt == "int8":
        v = q[:, i]
        el = torch.where(v > 127, v - 256, v).double() / 64
    else:
        bits = FORMATS[fmt][4]
        v = q[:, i] if bits == 8 else q[:, i // 2] >> (4 * (i % 2)) & 15
        sign = 1.0 - 2.0 * (v >> (bits - 1)).double()
        grid = _grid(fmt)
        el = sign * grid[(v & (2 ** (bits - 1) - 1)).clamp(max=grid.numel() - 1)]
    return el * torch.exp2(e.double())
