"""An MLP half of a block as it is used: two column-parallel products of which one is the other's gate, a row-parallel one, and the join
with its norms, dropout and the next block's input; forward and backward, eager, captured and on other streams."""
import numpy as np
import pytest
import torch

import act_util as au
from test_gpu_act import OFFSET, SEED, TORCH, keep_of, rng_of, values

pytestmark = pytest.mark.gpu


class Block:
    """Tensors of one block and its two passes; features of the MLP are pruned by one list (columns of the first products, the
    contraction of the second)."""

    def __init__(self, M, H, F, dtype, ratio, seed=0):
        from paper_2401_11469_amd import zr
        g = np.random.default_rng(seed)
        dt = TORCH[dtype]
        gpu = lambda *s, size=1.0: torch.from_numpy(values(g, dtype, *s, size=size)).to(dt).cuda()      # noqa: E731
        self.M, self.H, self.F, self.dt = M, H, F, dt
        self.x, self.h = gpu(M, H), gpu(M, H)
        self.Wg, self.Wu, self.Wd = gpu(F, H, size=H ** -0.5), gpu(F, H, size=H ** -0.5), gpu(F, H, size=F ** -0.5)
        self.bg, self.bd = gpu(F, size=0.1), gpu(H, size=0.1)
        self.post_w, self.pre_w, self.scale_v = gpu(H), gpu(H), gpu(H)
        self.keep = torch.from_numpy(keep_of(g, F, ratio).astype(np.int32)).cuda() if ratio else None
        self.dx, self.dh = gpu(M, H), gpu(M, H)
        self.rng = rng_of()
        new = lambda *s: torch.empty(s, dtype=dt, device="cuda")       # noqa: E731
        self.out = dict(U=new(M, F), Z=new(M, F), A=new(M, F), y=new(M, H), x1=new(M, H), h1=new(M, H),
                        dres=new(M, H), dy=new(M, H), dA=new(M, F), dWd=new(F, H), dha=new(M, H), dhb=new(M, H), dWg=new(F, H), dWu=new(F, H), dU=new(M, F),
                        dbg=new(F), dbd=new(H), dpost=new(H), dpre=new(H), dgate=new(H))
        n = self.keep.numel() if ratio else F
        size = max(zr.act_workspace_bytes(M, H, F, n, zr.DROP_N, dt, True), zr.act_workspace_bytes(M, F, H, n, zr.DROP_K, dt, True),
                   zr.block_join_workspace_bytes(M, H))
        self.ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def run(self, stream=None):
        from paper_2401_11469_amd import zr
        o, n = self.out, dict(keep_idx=self.keep, mode=zr.DROP_N, w_layout=zr.W_NK, workspace=self.ws, stream=stream)
        k = dict(keep_idx=self.keep, mode=zr.DROP_K, w_layout=zr.W_KN, workspace=self.ws, stream=stream)
        how = dict(norm=zr.NORM_RMS, post=True, pre=True, eps=1e-5, p=0.1, rng=self.rng, scale=0.5, bias=self.bd, gate=self.scale_v, post_w=self.post_w, pre_w=self.pre_w, stream=stream)
        zr.resized_linear_act_fwd(self.h, self.Wu, Y=o["U"], **n)
        zr.resized_linear_act_fwd(self.h, self.Wg, bias=self.bg, act=zr.ACT_SILU, gate=o["U"], Z=o["Z"], Y=o["A"], **n)
        zr.resized_linear_act_fwd(o["A"], self.Wd, Y=o["y"], **k)
        zr.block_join_fwd(o["y"], self.x, x_out=o["x1"], h=o["h1"], **how)
        # backward
        zr.block_join_bwd(self.dx, self.dh, o["x1"], o["y"], dx=o["dres"], dy=o["dy"], dbias=o["dbd"], dgate=o["dgate"], dpost_w=o["dpost"],
                          dpre_w=o["dpre"], workspace=self.ws, **how)
        zr.resized_linear_act_bwd(o["A"], self.Wd, o["dy"], dX=o["dA"], dW=o["dWd"], **k)
        zr.resized_linear_act_bwd(self.h, self.Wg, o["dA"], act=zr.ACT_SILU, Z=o["Z"], gate=o["U"], dX=o["dha"], dW=o["dWg"], dbias=o["dbg"], dgate=o["dU"], **n)
        zr.resized_linear_act_bwd(self.h, self.Wu, o["dU"], dX=o["dhb"], dW=o["dWu"], **n)
        return o

    def exact(self):
        """The same in 64 bits on the CPU, gradients by automatic differentiation."""
        d = {n: getattr(self, n).double().cpu().requires_grad_() for n in ("x", "h", "Wg", "Wu", "Wd", "bg", "bd", "post_w", "pre_w", "scale_v")}
        mask = torch.zeros(self.F, dtype=torch.float64)
        mask[self.keep.long().cpu() if self.keep is not None else slice(None)] = 1
        seed, offset = (int(v) & (2 ** 64 - 1) for v in self.rng.cpu())
        f = torch.from_numpy(au.factor(seed, offset, self.M, self.H, 0.1))
        U = (d["h"] @ d["Wu"].t()) * mask
        Z = (d["h"] @ d["Wg"].t()) * mask + d["bg"]
        A = Z * torch.sigmoid(Z) * U
        y = (A * mask) @ (d["Wd"] * mask[:, None])
        norm = lambda v: v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-5)      # noqa: E731
        x1 = d["x"] + 0.5 * d["scale_v"] * norm((y + d["bd"]) * f) * d["post_w"]
        h1 = norm(x1) * d["pre_w"]
        ((x1 * self.dx.double().cpu()).sum() + (h1 * self.dh.double().cpu()).sum()).backward()
        g = {n: t.grad for n, t in d.items()}
        return dict(y=y, x1=x1, h1=h1, dres=g["x"], dWg=g["Wg"], dWu=g["Wu"], dWd=g["Wd"], dbg=g["bg"], dbd=g["bd"], dpost=g["post_w"], dpre=g["pre_w"], dgate=g["scale_v"]), g["h"]


def far(a, b):
    return float((a.double().cpu() - b).norm() / b.norm())


@pytest.mark.parametrize("M,H,F,ratio", [(60, 96, 200, 0.25), (9, 136, 264, 0.0), (130, 512, 1408, 0.3)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_block_against_automatic_differentiation(M, H, F, ratio, dtype):
    b = Block(M, H, F, dtype, ratio)
    o = b.run()
    torch.cuda.synchronize()
    want, dh = b.exact()
    # relative distance of whole tensors.  At most a dozen values on the way to a result are rounded to its type, each by at most u
    # of itself and u / sqrt(3) at random, passed on by products without growing: sqrt(12 / 3) u, with a factor of two for the
    # norms, which pass on an error beside the value it came from; fp32 sums add sqrt(1500) 2^-24 a product.
    tol = 4 * au.U[dtype] + 8 * (4 * 1500 ** 0.5) * au.F
    for n, w in want.items():
        assert far(o[n], w.detach()) <= tol, (n, far(o[n], w.detach()), tol)
    assert far(o["dha"].double() + o["dhb"].double(), dh) <= tol


def test_block_in_a_graph_draws_anew_and_repeats():
    """Captured once, replayed with other seeds between eager work and synchronizations: every replay gives what an eager run gives."""
    for dtype, M, H, F, ratio in (("bf16", 300, 512, 1408, 0.25), ("f32", 40, 96, 200, 0.0), ("bf16", 7, 256, 768, 0.25)):
        b = Block(M, H, F, dtype, ratio)
        b.run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            b.run()
        for i in range(4):
            b.rng += 1 + i
            for t in b.out.values():
                t.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            got = {n: t.clone() for n, t in b.out.items()}
            b.run()
            torch.cuda.synchronize()
            for n, t in b.out.items():
                assert torch.equal(got[n], t), (dtype, i, n)


def test_two_graphs_that_share_a_workspace():
    a, b = Block(200, 256, 512, "bf16", 0.25, seed=1), Block(200, 256, 512, "bf16", 0.25, seed=2)
    b.ws = a.ws
    graphs, want = [], []
    for x in (a, b):
        x.run()
        torch.cuda.synchronize()
        want.append({n: t.clone() for n, t in x.out.items()})
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.run()
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    for x, w in zip((a, b), want):
        for n, t in x.out.items():
            assert torch.equal(t, w[n]), n


def test_two_streams_at_once():
    blocks = [Block(260, 256, 768, "bf16", 0.25, seed=s) for s in range(3)]
    want = []
    for b in blocks:
        b.run()
        torch.cuda.synchronize()
        want.append({n: t.clone() for n, t in b.out.items()})
    streams = [torch.cuda.Stream() for _ in blocks]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        for b, s in zip(blocks, streams):
            b.run(stream=s)
    torch.cuda.synchronize()
    for b, w in zip(blocks, want):
        for n, t in b.out.items():
            assert torch.equal(t, w[n]), n


def test_a_padded_batch_keeps_what_lies_behind_it():
    """Rows behind the last sequence are no rows of the call: they stay as they are."""
    from paper_2401_11469_amd import zr
    g = np.random.default_rng(3)
    M, rows, K, N = 24, 17, 64, 96
    X, W, G = (torch.from_numpy(values(g, "bf16", *s)).bfloat16().cuda() for s in ((M, K), (N, K), (M, N)))
    Y = torch.full((M, N), 3.25, dtype=torch.bfloat16, device="cuda")
    Z = Y.clone()
    zr.resized_linear_act_fwd(X[:rows], W, mode=zr.DROP_N, w_layout=zr.W_NK, act=zr.ACT_SILU, gate=G[:rows], Y=Y[:rows], Z=Z[:rows])
    assert (Y[rows:] == 3.25).all() and (Z[rows:] == 3.25).all()
    x1, h1 = torch.full((M, N), 3.25, dtype=torch.bfloat16, device="cuda"), torch.full((M, N), 3.25, dtype=torch.bfloat16, device="cuda")
    zr.block_join_fwd(G[:rows], G[:rows], x_out=x1[:rows], h=h1[:rows])
    assert (x1[rows:] == 3.25).all() and (h1[rows:] == 3.25).all()
    d = torch.full((M, K), 3.25, dtype=torch.bfloat16, device="cuda")
    zr.resized_linear_act_bwd(X[:rows], W, G[:rows], mode=zr.DROP_N, w_layout=zr.W_NK, act=zr.ACT_SILU, Z=Z[:rows], dX=d[:rows])
    assert (d[rows:] == 3.25).all() and d[:rows].isfinite().all()


def test_which_kernels_run():
    """The rules on sizes and types send each kind of call where it is meant to go."""
    from paper_2401_11469_amd import zr
    zr.debug_record_kernel_names(True)
    try:
        def name(M, K, N, keep=None, mode=1, w_layout=0, ws=False, dt=torch.bfloat16, off=0):
            X = torch.zeros(M * K + off, dtype=dt, device="cuda")[off:].view(M, K)
            W = torch.zeros((K, N) if w_layout == 0 else (N, K), dtype=dt, device="cuda")
            work = torch.empty(zr.act_workspace_bytes(M, K, N, keep.numel() if keep is not None else N, mode, dt), dtype=torch.uint8, device="cuda") if ws else None
            zr.resized_linear_act_fwd(X, W, keep, mode, w_layout=w_layout, workspace=work)
            return zr.debug_last_kernel()
        half = torch.arange(0, 2048, 2, dtype=torch.int32, device="cuda")
        assert name(1, 2048, 2048, mode=0, w_layout=1).startswith("act_few_rows_kernel<4")
        assert name(4, 2048, 2048, mode=0, w_layout=1).startswith("act_few_rows_kernel<8")
        assert name(16, 2048, 2048, half, mode=0, w_layout=1).startswith("act_few_rows_kernel<16")
        assert name(16, 2048, 2048).startswith("act_few_cols_kernel<false")
        assert name(3, 2048, 2048, half).startswith("act_few_cols_kernel<true")
        assert name(16, 2048, 2048, half, ws=True).startswith("act_few_cols_kernel<false")
        assert name(17, 2048, 2048).startswith("act_kernel<P, Q")
        assert name(8192, 1024, 2048, mode=0, w_layout=1).startswith("act_fast_kernel<RingP, RingP")
        assert name(8192, 2048, 2048, half, ws=True).startswith("act_fast_kernel<RingP, RingQM")
        assert "split" in name(256, 4096, 512, mode=0, w_layout=1, ws=True)
        assert name(8192, 64, 2064, mode=0, w_layout=1) == "act_kernel<P, P, 32, 256>"           # 16 columns behind a panel of whole rounds
        assert name(8192, 1032, 1024, off=1).startswith("act_kernel<P, Q")
        assert name(300, 256, 512, dt=torch.float32).startswith("f32_act_kernel<")
    finally:
        zr.debug_record_kernel_names(False)
