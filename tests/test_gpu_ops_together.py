"""The operators as a program uses them together: the router's outputs feed the
balance loss (and its gradient the router's weights) and, as expert_offsets and
pair_order, a SwiGLU FFN over experts held in FP8: quantize the tokens, the
grouped gate/up product over gathered rows, SwiGLU quantized, the grouped down
product, the weighted combine.  Every step against 64 bits, then the chain
captured into a graph and replayed on other tokens."""
import numpy as np
import pytest
import torch

import paper_2609_38090_amd as mira
from ops_reference import U32, balance, dequantize, gemm, gemm_bound, source_rows

pytestmark = pytest.mark.gpu
EPS = 1e-8


def _pad(n):
    return -(-n // 16) * 16


def _blk(n):
    return -(-n // 128)


class Fp8Layer:
    """A MoE layer whose experts are held in FP8 (gate over up, and down), beside the routing of the library."""

    def __init__(self, T, C, R, E, k, S, seed=0):
        self.T, self.C, self.R, self.E, self.k, self.S = T, C, R, E, k, S
        G, P = E + S, T * k + S * T
        self.G, self.P = G, P
        g = torch.Generator(device="cuda").manual_seed(seed)
        rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.x = rn(T, C).bfloat16()
        self.wr = (rn(E, C) / C ** 0.5).bfloat16()
        self.bias = -torch.log(torch.arange(1, E + 1, device="cuda", dtype=torch.float32))
        u8 = lambda *s: torch.empty(*s, dtype=torch.uint8, device="cuda")  # noqa: E731
        f32 = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
        self.w1, self.s1 = u8(G, 2 * R, _pad(C)), f32(G, _blk(2 * R), _blk(C))
        self.w2, self.s2 = u8(G, C, _pad(R)), f32(G, _blk(C), _blk(R))
        for e in range(G):
            for w, s, rows, cols in ((self.w1, self.s1, 2 * R, C), (self.w2, self.s2, C, R)):
                mira.mira_fp8_quantize(mira.Fp8QuantArgs(x=rn(rows, cols) * 0.02, x_dtype=mira.MIRA_F32, rows=rows, cols=cols,
                                                         block_rows=128, eps=EPS, q=w[e], scale=s[e]))
        torch.cuda.synchronize()
        i32 = lambda *s: torch.empty(*s, dtype=torch.int32, device="cuda")  # noqa: E731
        self.shape = mira.MoEShape(C, R, E, k, S, mira.MIRA_BF16)
        stride = mira.mira_packed_expert_bytes(C, R)
        nb = mira.mira_workspace_bytes(self.shape, T)
        self.route = mira.MoEArgs(
            x=self.x, n_tokens=T, n_slots=G, w_router=self.wr, router_bias=self.bias,
            slot_table=torch.arange(G, dtype=torch.int32, device="cuda"), slot_pool=u8(G * stride), slot_stride=stride,
            out=f32(T, C), topk_idx=i32(T, k), topk_weight=f32(T, k), logits=f32(T, E), expert_counts=i32(G),
            expert_offsets=i32(G + 1), pair_order=i32(P), workspace=u8(nb), workspace_bytes=nb)
        self.bal = dict(loss=f32(1), counts=i32(1, E), mean_prob=f32(1, E), dlogits=f32(T, E))
        nb = mira.mira_balance_workspace_bytes(T, E)
        self.balance = mira.BalanceArgs(logits=self.route.logits, topk_idx=self.route.topk_idx, n_tokens=T, n_experts=E, top_k=k,
                                        coef=0.5, workspace=u8(nb), workspace_bytes=nb, **self.bal)
        self.xq, self.xs = u8(T, _pad(C)), f32(T, _blk(C))
        self.quant_x = mira.Fp8QuantArgs(x=self.x, rows=T, cols=C, eps=EPS, q=self.xq, scale=self.xs)
        self.h = torch.empty(P, 2 * R, dtype=torch.bfloat16, device="cuda")
        self.hq, self.hs = u8(P, _pad(R)), f32(P, _blk(R))
        self.quant_h = mira.Fp8QuantArgs(x=self.h, rows=P, cols=R, eps=EPS, flags=mira.MIRA_FP8_SWIGLU, q=self.hq, scale=self.hs)
        self.y = f32(P, C)
        self.gate_up = mira.Fp8GemmArgs(m=P, n=2 * R, k=C, n_groups=G, out_dtype=mira.MIRA_BF16, x_rows=T, top_k=k, x=self.xq,
                                        x_scale=self.xs, w=self.w1, w_scale=self.s1, offsets=self.route.expert_offsets,
                                        pair_order=self.route.pair_order, out=self.h)
        self.down = mira.Fp8GemmArgs(m=P, n=C, k=R, n_groups=G, out_dtype=mira.MIRA_F32, x_rows=P, x=self.hq, x_scale=self.hs,
                                     w=self.w2, w_scale=self.s2, offsets=self.route.expert_offsets, out=self.y)
        for a in (self.gate_up, self.down):
            nb = mira.mira_fp8_gemm_workspace_bytes(a)
            a.workspace, a.workspace_bytes = u8(nb), nb

    def run(self):
        mira.mira_moe_route(self.shape, self.route)
        mira.mira_balance_loss(self.balance)
        mira.mira_fp8_quantize(self.quant_x)
        mira.mira_fp8_gemm(self.gate_up)
        mira.mira_fp8_quantize(self.quant_h)
        mira.mira_fp8_gemm(self.down)
        # combine: pair p < T k has its token's weight, a shared pair 1
        p = self.route.pair_order.long()
        tok = source_rows(p, self.T, self.k)
        wt = torch.where(p < self.T * self.k, self.route.topk_weight.reshape(-1)[p.clamp(max=self.T * self.k - 1)], 1.0)
        self.tok, self.wt = tok, wt
        self.out = torch.zeros(self.T, self.C, device="cuda").index_add_(0, tok, self.y * wt[:, None])
        return self.out

    def check(self):
        T, C, R, E, k, G, P = self.T, self.C, self.R, self.E, self.k, self.G, self.P
        idx = self.route.topk_idx.cpu().numpy()
        loss, counts, mean, d = balance(self.route.logits.double().cpu().numpy(), idx, np.array([0, T]), np.ones(T, np.uint8), 0.5, np.ones(1))
        assert np.array_equal(self.bal["counts"].cpu().numpy(), counts)
        assert np.array_equal(counts[0], self.route.expert_counts.cpu().numpy()[:E])
        assert abs(float(self.bal["loss"]) - loss[0]) <= 1000 * U32 * loss[0]      # sums of at most 300 terms, exp at 2 steps
        assert np.abs(self.bal["dlogits"].cpu().numpy() - d).max() <= 100 * U32 * 0.5 / T * counts.max() * E / (k * T)
        off = self.route.expert_offsets.tolist()
        x = dequantize(self.xq, self.xs, 1, T, C)
        h, hq = self.h.double().cpu(), dequantize(self.hq, self.hs, 1, P, R)
        y = self.y.double().cpu()
        for g in range(G):
            a, b = off[g], off[g + 1]
            if a == b:
                continue
            want, mag = gemm(x[self.tok[a:b]], dequantize(self.w1[g], self.s1[g], 128, 2 * R, C))
            assert ((h[a:b] - want).abs() <= gemm_bound(mag, C, True, want)).all()
            want, mag = gemm(hq[a:b], dequantize(self.w2[g], self.s2[g], 128, C, R))
            assert ((y[a:b] - want).abs() <= gemm_bound(mag, R, False, want)).all()
        act = torch.nn.functional.silu(h[:, :R]) * h[:, R:]
        sc = self.hs.double().cpu().repeat_interleave(128, 1)[:, :R]
        assert ((hq.cpu() - act).abs() <= (2.0 ** -4 * (1 + 2.0 ** -10) + 12 * U32) * act.abs() + 2.0 ** -10 * sc).all()
        want = torch.zeros(T, C, dtype=torch.float64).index_add_(0, self.tok.cpu(), y * self.wt.double().cpu()[:, None])
        assert float((self.out.double().cpu() - want).abs().max()) <= (k + self.S + 2) * U32 * float((y.abs().max() * (k + self.S)))


@pytest.mark.parametrize("T,C,R,E,k,S", [(1, 256, 384, 8, 2, 0), (16, 256, 192, 16, 4, 1), (300, 320, 448, 12, 3, 2), (700, 512, 256, 4, 2, 0)])
def test_layer_of_fp8_experts(T, C, R, E, k, S):
    lay = Fp8Layer(T, C, R, E, k, S)
    lay.run()
    torch.cuda.synchronize()
    lay.check()


@pytest.mark.parametrize("T", [5, 300])
def test_graph_replays_on_other_tokens(T):
    lay = Fp8Layer(T, 320, 448, 12, 3, 1)
    lay.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lay.run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lay.run()
    captured = lay.out
    for seed in range(4):
        lay.x.copy_(torch.randn(T, 320, generator=torch.Generator(device="cuda").manual_seed(100 + seed), device="cuda").bfloat16())
        eager = lay.run().clone()          # eager work on the same buffers between the replays
        torch.cuda.synchronize()
        captured.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        lay.out = captured
        lay.check()
        assert torch.allclose(captured, eager, rtol=0, atol=float(eager.abs().max()) * 2e-6)   # index_add_'s order


def test_router_gradient_from_the_loss():
    """The balance loss's gradient taken to the router's weights against central
    differences of the 64-bit loss (counts held constant)."""
    lay = Fp8Layer(200, 256, 128, 8, 2, 0)
    lay.run()
    torch.cuda.synchronize()
    dw = (lay.bal["dlogits"].double().t() @ lay.x.double()).cpu()
    x, wr, bias = lay.x.double().cpu().numpy(), lay.wr.double().cpu().numpy(), lay.bias.double().cpu().numpy()
    idx = lay.route.topk_idx.cpu().numpy()

    def loss(w):
        return balance(x @ w.T + bias, idx, np.array([0, lay.T]), np.ones(lay.T, np.uint8), 0.5, np.ones(1))[0][0]

    h = 1e-4
    for e, c in ((0, 0), (3, 77), (7, 255)):
        a, b = wr.copy(), wr.copy()
        a[e, c] += h
        b[e, c] -= h
        want = (loss(a) - loss(b)) / (2 * h)
        # third derivative along one weight: at most coef max f mean |x|^3; logits in fp32 with bf16 products
        f = lay.bal["counts"].max().item() * lay.E / (lay.k * lay.T)
        tol = h * h * 0.5 * f * float(np.mean(np.abs(x[:, c]) ** 3)) + 1e-5 * 0.5 * f * float(np.mean(np.abs(x[:, c]))) + 4 * 2.0 ** -52 / h
        assert abs(float(dw[e, c]) - want) <= tol
