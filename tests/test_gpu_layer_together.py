"""A layer of FP8 experts from residual stream to residual stream and back, as a
training step with frozen experts runs it: norm with the residual's addition, the
router's logits, selection by sigmoid scores with a bias, groups and a mask, the
balance loss, the grouped gate/up product over gathered rows, SwiGLU, the grouped down
product, the combine; then the combine's gradient, the products on transposed copies,
SwiGLU's gradient, the gradient of gathering, of the selection and of the norm.
Every step against 64 bits of its own inputs, the whole against 64-bit gradients
of the unquantised layer, then captured and replayed on other tokens; streams."""
import numpy as np
import pytest
import torch

import paper_2609_38090_amd as mira
from layer_reference import U16, U32, f64, norm, norm_grad, pairs, select, select_grad, swiglu_grad
from ops_reference import dequantize, gemm, gemm_bound

pytestmark = pytest.mark.gpu
EPS, Q_EPS = 1e-6, 1e-8


def _pad(n):
    return -(-n // 16) * 16


def _blk(n):
    return -(-n // 128)


class Layer:
    def __init__(self, T, C, R, E, k, S, groups, top, masked, seed=0):
        self.T, self.C, self.R, self.E, self.k, self.S = T, C, R, E, k, S
        self.groups, self.top = groups, top
        G, P = E + S, T * (k + S)
        self.G, self.P = G, P
        g = torch.Generator(device="cuda").manual_seed(seed)
        rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        u8 = lambda *s: torch.empty(*s, dtype=torch.uint8, device="cuda")  # noqa: E731
        f32 = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
        i32 = lambda *s: torch.empty(*s, dtype=torch.int32, device="cuda")  # noqa: E731
        b16 = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        F, B = mira.MIRA_F32, mira.MIRA_BF16
        self.x, self.res = rn(T, C).bfloat16(), rn(T, C).bfloat16()
        self.dout = (0.1 * rn(T, C)).bfloat16()
        self.wn = (1 + 0.1 * rn(C)).bfloat16()
        self.wr = (rn(E, C) / C ** 0.5).bfloat16()
        self.bias = 0.2 * rn(E)
        self.mask = (torch.rand(T, generator=g, device="cuda") < 0.8).to(torch.uint8) if masked else None
        self.w = {}
        for name, rows, cols in (("w1", 2 * R, C), ("w2", C, R)):
            q, s, qt, st = u8(G, rows, _pad(cols)), f32(G, _blk(rows), _blk(cols)), u8(G, cols, _pad(rows)), f32(G, _blk(cols), _blk(rows))
            for e in range(G):
                mira.mira_fp8_quantize(mira.Fp8QuantArgs(x=rn(rows, cols) / cols ** 0.5, x_dtype=F, rows=rows, cols=cols, block_rows=128, eps=Q_EPS, q=q[e],
                                                         scale=s[e], qt=qt[e], scale_t=st[e]))
            torch.cuda.synchronize()
            self.w[name] = (q, s, qt, st)
        self.sum, self.y, self.xq, self.xs = b16(T, C), b16(T, C), u8(T, _pad(C)), f32(T, _blk(C))
        self.norm = mira.RmsNormArgs(x=self.x, residual=self.res, weight=self.wn, rows=T, cols=C, eps=EPS, q_eps=Q_EPS, sum=self.sum, y=self.y, q=self.xq,
                                     scale=self.xs)
        stride = mira.mira_packed_expert_bytes(C, 64)
        self.shape = mira.MoEShape(C, 64, E, k, 0, B)
        nb = mira.mira_workspace_bytes(self.shape, T)
        self.logits = f32(T, E)   # (the routing call's; the selection here is another)
        self.fused = mira.MoEArgs(x=self.y, n_tokens=T, n_slots=1, w_router=self.wr, slot_table=i32(E).zero_(), slot_pool=u8(stride).zero_(), slot_stride=stride,
                                  out=f32(T, C), logits=self.logits, workspace=u8(nb), workspace_bytes=nb)
        self.flags = mira.MIRA_ROUTE_SIGMOID | mira.MIRA_ROUTE_RENORM
        self.idx, self.weight, self.counts, self.offsets, self.order, self.pos = i32(T, k), f32(T, k), i32(G), i32(G + 1), i32(P), i32(P)
        nb = mira.mira_route_select_workspace_bytes(T, E, k, S)
        self.select = mira.RouteSelectArgs(logits=self.logits, bias=self.bias, mask=self.mask, n_tokens=T, n_experts=E, top_k=k, n_shared=S, n_groups=groups,
                                           top_groups=top, group_best=2, flags=self.flags, scale=2.0, topk_idx=self.idx, topk_weight=self.weight,
                                           expert_counts=self.counts, expert_offsets=self.offsets, pair_order=self.order, pair_pos=self.pos, workspace=u8(nb),
                                           workspace_bytes=nb)
        nb = mira.mira_balance_workspace_bytes(T, E)
        self.loss, self.dbal = f32(1), f32(T, E)
        self.balance = mira.BalanceArgs(logits=self.logits, topk_idx=self.idx, mask=self.mask, n_tokens=T, n_experts=E, top_k=k, coef=0.01, loss=self.loss,
                                        dlogits=self.dbal, workspace=u8(nb), workspace_bytes=nb)
        # rows that no pair has are never written by the products: whatever they hold must not matter
        self.h, self.hq, self.hs, self.yp = b16(P, 2 * R).fill_(float("nan")), u8(P, _pad(R)), f32(P, _blk(R)), b16(P, C).fill_(float("nan"))
        self.gate_up = self._product(P, 2 * R, C, self.xq, self.xs, "w1", 0, self.h, T, order=self.order)
        self.quant_h = mira.Fp8QuantArgs(x=self.h, rows=P, cols=R, eps=Q_EPS, flags=mira.MIRA_FP8_SWIGLU, q=self.hq, scale=self.hs)
        self.down = self._product(P, C, R, self.hq, self.hs, "w2", 0, self.yp, P)
        self.out = b16(T, C)
        self.combine = mira.CombineArgs(y=self.yp, topk_weight=self.weight, pair_pos=self.pos, residual=self.sum, n_tokens=T, top_k=k, n_shared=S, cols=C, y_rows=P,
                                        out=self.out)
        # back
        self.dyq, self.dys, self.dweight = u8(P, _pad(C)).zero_(), f32(P, _blk(C)).zero_(), f32(T, k)
        self.combine_grad = mira.CombineGradArgs(dout=self.dout, y=self.yp, topk_weight=self.weight, pair_pos=self.pos, n_tokens=T, top_k=k, n_shared=S, cols=C,
                                                 y_rows=P, q_eps=Q_EPS, q=self.dyq, scale=self.dys, dweight=self.dweight)
        self.dact = b16(P, R).fill_(float("nan"))
        self.down_t = self._product(P, R, C, self.dyq, self.dys, "w2", 2, self.dact, P)
        self.dhq, self.dhs = u8(P, _pad(2 * R)), f32(P, _blk(2 * R))
        self.swiglu = mira.SwigluGradArgs(x=self.h, dact=self.dact, rows=P, cols=R, q_eps=Q_EPS, q=self.dhq, scale=self.dhs)
        self.dxp = f32(P, C).fill_(float("nan"))
        self.up_t = self._product(P, C, 2 * R, self.dhq, self.dhs, "w1", 2, self.dxp, P, out_dtype=F)
        self.dy = f32(T, C)
        self.gather = mira.CombineArgs(y=self.dxp, pair_pos=self.pos, n_tokens=T, top_k=k, n_shared=S, cols=C, y_rows=P, y_dtype=F, out_dtype=F, out=self.dy)
        self.dlogits = f32(T, E)
        self.select_grad = mira.RouteSelectGradArgs(logits=self.logits, topk_idx=self.idx, dweight=self.dweight, add=self.dbal, n_tokens=T, n_experts=E, top_k=k,
                                                    flags=self.flags, scale=2.0, dlogits=self.dlogits)
        nb = mira.mira_rmsnorm_grad_workspace_bytes(T, C)
        self.dx, self.dwn = b16(T, C), f32(C)
        self.norm_grad = mira.RmsNormGradArgs(dy=self.dy, dsum=self.dout, h=self.sum, weight=self.wn, y_dtype=F, rows=T, cols=C, eps=EPS, dx=self.dx,
                                              dweight=self.dwn, workspace=u8(nb), workspace_bytes=nb)

    def _product(self, m, n, k, x, xs, name, copy, out, x_rows, order=None, out_dtype=mira.MIRA_BF16):
        w = self.w[name]
        a = mira.Fp8GemmArgs(m=m, n=n, k=k, n_groups=self.G, out_dtype=out_dtype, x_rows=x_rows, top_k=self.k if order is not None else 0, x=x, x_scale=xs,
                             w=w[copy], w_scale=w[copy + 1], offsets=self.offsets, pair_order=order, out=out)
        nb = mira.mira_fp8_gemm_workspace_bytes(a)
        a.workspace, a.workspace_bytes = torch.empty(nb, dtype=torch.uint8, device="cuda"), nb
        return a

    def forward(self):
        mira.mira_rmsnorm(self.norm)
        mira.mira_moe_route(self.shape, self.fused)
        mira.mira_route_select(self.select)
        mira.mira_balance_loss(self.balance)
        mira.mira_fp8_gemm(self.gate_up)
        mira.mira_fp8_quantize(self.quant_h)
        mira.mira_fp8_gemm(self.down)
        mira.mira_combine(self.combine)

    def backward(self):
        mira.mira_combine_grad(self.combine_grad)
        mira.mira_fp8_gemm(self.down_t)
        mira.mira_swiglu_grad(self.swiglu)
        mira.mira_fp8_gemm(self.up_t)
        mira.mira_combine(self.gather)
        mira.mira_route_select_grad(self.select_grad)
        mira.mira_rmsnorm_grad(self.norm_grad)

    def step(self):
        self.forward()
        self.backward()

    def results(self):
        live = int(self.offsets[-1])
        return [t.clone() for t in (self.sum, self.y, self.idx, self.weight, self.counts, self.offsets, self.order, self.pos, self.h[:live], self.yp[:live], self.out,
                                    self.loss, self.dyq[:live], self.dweight, self.dact[:live], self.dhq[:live], self.dy, self.dlogits, self.dx, self.dwn)]

    def check(self):
        T, C, R, E, k, S, G, P = self.T, self.C, self.R, self.E, self.k, self.S, self.G, self.P
        mask = None if self.mask is None else self.mask.cpu().numpy()
        h = self.x + self.res
        assert torch.equal(self.sum, h)
        y, _ = norm(f64(h), f64(self.wn), EPS)
        assert (np.abs(f64(self.y) - y) <= (U16 + 60 * U32) * np.abs(y)).all()
        idx, w = select(f64(self.logits), k, True, True, f64(self.bias), mask, self.groups, self.top, 2, 2.0)
        assert np.array_equal(self.idx.cpu().numpy(), idx)
        assert (np.abs(f64(self.weight) - w) <= 64 * U32 * w).all()
        counts, offsets, order, pos = pairs(idx, mask, E, S)
        for got, want in zip((self.counts, self.offsets, self.order, self.pos), (counts, offsets, order, pos)):
            assert np.array_equal(got.cpu().numpy(), want)
        live = int(offsets[-1])
        tok = np.where(order[:live] < T * k, order[:live] // k, (order[:live] - T * k) % T)
        # products: the operands as they are held
        group = np.repeat(np.arange(G), counts)

        def held(name, copy, e, rows, cols):
            q, s = self.w[name][copy][e], self.w[name][copy + 1][e]
            return dequantize(q, s, 128, rows, cols).cpu()

        for x, xs, cols, name, copy, n, got, src, bf16 in (
                (self.xq, self.xs, C, "w1", 0, 2 * R, self.h, tok, True), (self.hq, self.hs, R, "w2", 0, C, self.yp, np.arange(live), True),
                (self.dyq, self.dys, C, "w2", 2, R, self.dact, np.arange(live), True), (self.dhq, self.dhs, 2 * R, "w1", 2, C, self.dxp, np.arange(live), False)):
            values = dequantize(x, xs, 1, x.shape[0], cols).cpu()
            for e in range(G):
                at = np.nonzero(group == e)[0]
                if len(at):
                    want, mag = gemm(values[src[at]], held(name, copy, e, n, cols))
                    assert ((got[:live].double().cpu()[at] - want).abs() <= gemm_bound(mag, cols, bf16, want)).all(), name
        wt = np.concatenate([f64(self.weight), np.ones((T, S))], 1)
        at = np.concatenate([pos[:T * k].reshape(T, k), pos[T * k:].reshape(S, T).T], 1)
        has = at >= 0
        rows = np.where(has[:, :, None], f64(self.yp)[np.maximum(at, 0)], 0.0)
        want, mag = (rows * wt[:, :, None]).sum(1) + f64(self.sum), (np.abs(rows) * wt[:, :, None]).sum(1) + np.abs(f64(self.sum))
        assert (np.abs(f64(self.out) - want) <= U16 * np.abs(want) + (k + S + 2) * 2 * U32 * mag).all()
        d = f64(self.dout)
        prod = rows[:, :k] * d[:, None, :]
        assert (np.abs(f64(self.dweight) - prod.sum(2)) <= (8 * -(-C // 2048) + 12) * U32 * np.abs(prod).sum(2)).all()
        dyp = np.zeros((live, C))
        for j in range(k + S):
            dyp[at[has[:, j], j]] = d[has[:, j]] * wt[has[:, j], j][:, None]
        got = dequantize(self.dyq, self.dys, 1, P, C).cpu().numpy()[:live]
        scale = np.repeat(self.dys.cpu().numpy()[:live], 128, 1)[:, :C]
        assert (np.abs(got - dyp) <= (2.0 ** -4 + 20 * U32) * np.abs(dyp) + 2.0 ** -10 * scale).all()
        dg, du, mag = swiglu_grad(f64(self.h)[:live, :R], f64(self.h)[:live, R:], f64(self.dact)[:live])
        dh, mag = np.concatenate([dg, du], 1), np.concatenate([mag, np.abs(du)], 1)
        got = dequantize(self.dhq, self.dhs, 1, P, 2 * R).cpu().numpy()[:live]
        scale = np.repeat(self.dhs.cpu().numpy()[:live], 128, 1)[:, :2 * R]
        assert (np.abs(got - dh) <= 2.0 ** -4 * np.abs(dh) + 2.0 ** -10 * scale + 60 * U32 * mag).all()
        rows = np.where(has[:, :, None], f64(self.dxp)[np.maximum(at, 0)], 0.0)
        assert (np.abs(f64(self.dy) - rows.sum(1)) <= (k + S + 1) * U32 * np.abs(rows).sum(1)).all()
        dl, mag = select_grad(f64(self.logits), idx, f64(self.dweight), True, True, 2.0)
        dl, mag = dl + f64(self.dbal), mag + np.abs(f64(self.dbal))
        assert (np.abs(f64(self.dlogits) - dl) <= 128 * U32 * mag + 1e-37).all()
        dx, dw, terms, wmag = norm_grad(f64(self.dy), d, f64(self.sum), f64(self.wn), EPS)
        assert (np.abs(f64(self.dx) - dx) <= U16 * np.abs(dx) + 200 * U32 * terms).all()
        assert (np.abs(f64(self.dwn) - dw) <= (T + 100) * U32 * wmag).all()


CASES = [(1, 256, 128, 8, 2, 0, 2, 1, False), (16, 256, 192, 16, 4, 1, 4, 2, False), (300, 320, 200, 12, 3, 2, 3, 2, True), (700, 512, 256, 8, 2, 0, 4, 3, True)]


@pytest.mark.parametrize("case", CASES)
def test_every_step(case):
    lay = Layer(*case)
    lay.step()
    torch.cuda.synchronize()
    lay.check()


def test_gradients_of_the_whole():
    """Against 64-bit gradients of the layer without 8-bit rounding.  Each of the five operands held in e4m3 is off
    by at most 2^-4, in the mean by 2^-4 / sqrt(3) of each value, so five of them leave an angle of about 0.08
    between the gradients (cosine 0.997), and of 0.16 (0.987) if all added up."""
    lay = Layer(200, 512, 256, 8, 2, 1, 1, 1, False)
    lay.select.n_groups = lay.select.top_groups = 1
    lay.groups = lay.top = 1
    lay.step()
    torch.cuda.synchronize()
    T, C, R, E, k = lay.T, lay.C, lay.R, lay.E, lay.k
    x, wn = lay.sum.double().cpu().requires_grad_(), lay.wn.double().cpu().requires_grad_()
    y = x / torch.sqrt((x * x).mean(1, keepdim=True) + EPS) * wn
    logits = lay.logits.double().cpu().requires_grad_()
    sel = torch.sigmoid(logits).gather(1, lay.idx.long().cpu())
    weight = 2.0 * sel / (sel.sum(1, keepdim=True) + 1e-20)
    out = x * 1.0
    for e in range(E + 1):
        w1, w2 = (dequantize(lay.w[n][0][e], lay.w[n][1][e], 128, r, c).cpu() for n, r, c in (("w1", 2 * R, C), ("w2", C, R)))
        h = y @ w1.t()
        o = (torch.nn.functional.silu(h[:, :R]) * h[:, R:]) @ w2.t()
        share = torch.where(lay.idx.cpu() == e, weight, torch.zeros_like(weight)).sum(1) if e < E else torch.ones(T, dtype=torch.float64)
        out = out + share[:, None] * o
    gx, gw, gl = torch.autograd.grad(out, (x, wn, logits), lay.dout.double().cpu())

    def cosine(a, b):
        a, b = a.double().cpu().reshape(-1), b.double().cpu().reshape(-1)
        return float((a * b).sum() / (a.norm() * b.norm()))

    assert cosine(lay.out, out.detach()) > 0.99
    assert cosine(lay.dx, gx) > 0.987 and cosine(lay.dwn, gw) > 0.987 and cosine(lay.dlogits - lay.dbal, gl) > 0.987
    # without the residual's own share, which is exact
    assert cosine(lay.dx.double().cpu() - lay.dout.double().cpu(), gx - lay.dout.double().cpu()) > 0.987


@pytest.mark.parametrize("case", [CASES[1], CASES[2]])
def test_graph_replays_on_other_tokens(case):
    """Captured once, replayed on other tokens with eager work on the same buffers in between: the eager bits."""
    lay = Layer(*case)
    lay.step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lay.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lay.step()
    for seed in range(4):
        g = torch.Generator(device="cuda").manual_seed(50 + seed)
        lay.x.copy_(torch.randn(lay.T, lay.C, generator=g, device="cuda").bfloat16())
        lay.bias.copy_(0.2 * torch.randn(lay.E, generator=g, device="cuda"))
        if lay.mask is not None:
            lay.mask.copy_((torch.rand(lay.T, generator=g, device="cuda") < 0.7).to(torch.uint8))
        lay.step()
        torch.cuda.synchronize()
        eager = lay.results()
        for t in (lay.out, lay.dx, lay.dwn, lay.dlogits, lay.dweight, lay.weight):
            t.fill_(float("nan"))
        lay.idx.fill_(99)
        lay.pos.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, lay.results()):
            assert torch.equal(a, b)
        if seed == 0:
            lay.check()


def test_two_layers_on_two_streams_at_once():
    a, b = Layer(*CASES[2], seed=1), Layer(*CASES[3], seed=2)
    want = []
    for lay in (a, b):
        lay.step()
        torch.cuda.synchronize()
        want.append(lay.results())
        for t in (lay.out, lay.dx, lay.dwn, lay.dlogits):
            t.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for lay, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                lay.step()
    torch.cuda.synchronize()
    for lay, w in zip((a, b), want):
        for x, y in zip(w, lay.results()):
            assert torch.equal(x, y)


def test_gradients_with_the_router():
    """The gradient that reaches the norm's input and the router's matrix, the selection's and the balance loss's going through
    that matrix: the products with it are the caller's.  Bounds as of the whole without it."""
    lay = Layer(200, 512, 256, 8, 2, 1, 1, 1, False)
    lay.step()
    torch.cuda.synchronize()
    T, R, E = lay.T, lay.R, lay.E
    without = lay.dx.clone()
    lay.dy += lay.dlogits @ lay.wr.float()
    dwr = lay.dlogits.t().contiguous() @ lay.y.float()
    mira.mira_rmsnorm_grad(lay.norm_grad)
    torch.cuda.synchronize()
    x, wn, wr = (t.double().cpu().requires_grad_() for t in (lay.sum, lay.wn, lay.wr))
    y = x / torch.sqrt((x * x).mean(1, keepdim=True) + EPS) * wn
    logits = y @ wr.t()
    sel = torch.sigmoid(logits).gather(1, lay.idx.long().cpu())
    weight = 2.0 * sel / (sel.sum(1, keepdim=True) + 1e-20)
    out = x * 1.0
    for e in range(E + 1):
        w1, w2 = (dequantize(lay.w[n][0][e], lay.w[n][1][e], 128, r, c).cpu() for n, r, c in (("w1", 2 * R, lay.C), ("w2", lay.C, R)))
        h = y @ w1.t()
        o = (torch.nn.functional.silu(h[:, :R]) * h[:, R:]) @ w2.t()
        share = torch.where(lay.idx.cpu() == e, weight, torch.zeros_like(weight)).sum(1) if e < E else torch.ones(T, dtype=torch.float64)
        out = out + share[:, None] * o
    loss = (out * lay.dout.double().cpu()).sum() + (logits * lay.dbal.double().cpu()).sum()
    gx, gw, gr = torch.autograd.grad(loss, (x, wn, wr))

    def cosine(a, b):
        a, b = a.double().cpu().reshape(-1), b.double().cpu().reshape(-1)
        return float((a * b).sum() / (a.norm() * b.norm()))

    res = lay.dout.double().cpu()
    assert cosine(lay.dx.double().cpu() - res, gx - res) > 0.987 and cosine(lay.dwn, gw) > 0.987 and cosine(dwr, gr) > 0.987
    assert cosine(lay.dx, gx) > cosine(without, gx)
