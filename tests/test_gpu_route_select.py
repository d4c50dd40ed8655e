"""The selection of experts from logits, the pairs' order and the weights'
gradient against 64 bits: softmax and sigmoid scores, biases, groups, masks,
candidates that fp32 does not tell apart, ties, special logits."""
import numpy as np
import pytest
import torch

import paper_2609_38090_amd as mira
from layer_reference import TINY, U32, Guarded, code, dt, f64, pairs, scores, select, select_grad, unit

pytestmark = pytest.mark.gpu
# s: exp 4 half steps, 10 additions, the reciprocal 2, products; renormalised: 16 additions, a quotient, two products
STEPS = 64


class Call:
    def __init__(self, x, k, S=0, sigmoid=False, renorm=False, bias=None, mask=None, groups=1, top_groups=1, best=1, scale=1.0, pad=0, shift=0,
                 outs="wcofp"):
        T, E = x.shape
        self.T, self.E, self.k, self.S = T, E, k, S
        name = "f32" if x.dtype == torch.float32 else "bf16"
        self.X = Guarded(max(T, 1), E, x.dtype, E + pad, shift)
        if T:
            self.X.put(x)
        self.idx, self.w = Guarded(max(T, 1), k, torch.int32), Guarded(max(T, 1), k, torch.float32)
        P = T * (k + S)
        self.counts, self.offsets = Guarded(1, E + S, torch.int32), Guarded(1, E + S + 1, torch.int32)
        self.order, self.pos = Guarded(1, max(P, 1), torch.int32), Guarded(1, max(P, 1), torch.int32)
        nb = mira.mira_route_select_workspace_bytes(T, E, k, S)
        self.ws = Guarded(1, nb, torch.uint8)
        self.bias, self.mask = bias, mask
        self.opt = dict(sigmoid=sigmoid, renorm=renorm, groups=groups, top_groups=top_groups, best=best, scale=scale)
        self.args = mira.RouteSelectArgs(
            logits=self.X.v, bias=bias, mask=mask, logits_dtype=code(name), n_tokens=T, n_experts=E, top_k=k, n_shared=S, n_groups=groups,
            top_groups=top_groups, group_best=best, flags=(mira.MIRA_ROUTE_SIGMOID if sigmoid else 0) | (mira.MIRA_ROUTE_RENORM if renorm else 0),
            scale=scale, ld_logits=E + pad, topk_idx=self.idx.v, topk_weight=self.w.v if "w" in outs else None,
            expert_counts=self.counts.v if "c" in outs else None, expert_offsets=self.offsets.v if "o" in outs else None,
            pair_order=self.order.v if "f" in outs else None, pair_pos=self.pos.v if "p" in outs else None, workspace=self.ws.v, workspace_bytes=nb)

    def run(self, stream=None):
        mira.mira_route_select(self.args, stream)
        return self

    def outputs(self):
        T, P = self.T, self.T * (self.k + self.S)
        return [t.cpu().numpy() for t in (self.idx.v[:T], self.w.v[:T], self.counts.v[0], self.offsets.v[0], self.order.v[0, :P], self.pos.v[0, :P])]

    def check(self, rows=None, extra=0.0):
        torch.cuda.synchronize()
        guards = (self.X, self.idx, self.w, self.counts, self.offsets, self.order, self.pos, self.ws)
        assert all(g.intact() for g in guards)
        x = f64(self.X.v)[:self.T]
        mask = None if self.mask is None else self.mask.cpu().numpy()
        idx, weight = select(x, self.k, bias=None if self.bias is None else f64(self.bias), mask=mask, **self.opt)
        i, w, counts, offsets, order, pos = self.outputs()
        assert np.array_equal(i, idx)
        assert (np.abs(w - weight) <= STEPS * U32 * np.abs(weight) + 2.0 ** -120 + extra).all()
        for got, want in zip((counts, offsets, order, pos), pairs(idx, mask, self.E, self.S)):
            assert np.array_equal(got, want)
        return self


def _logits(rng, T, E, name):
    return torch.from_numpy(rng.normal(0, 1.5, (T, E)) - 0.5 * np.log(np.arange(1, E + 1))).cuda().to(dt(name))


@pytest.mark.parametrize("T,E,k,S", [(1, 1, 1, 0), (1, 8, 2, 0), (16, 8, 2, 0), (5, 64, 6, 2), (32, 3, 3, 1), (33, 100, 16, 0), (64, 256, 8, 0), (301, 61, 4, 3),
                                     (700, 128, 8, 1), (2048, 64, 6, 2), (9000, 5, 2, 0)])
@pytest.mark.parametrize("sigmoid,renorm,biased,masked,name,pad,shift", [
    (False, True, False, False, "f32", 0, 0), (True, True, True, True, "f32", 3, 1), (False, False, True, False, "bf16", 0, 0),
    (True, False, False, True, "bf16", 5, 3), (False, True, True, True, "bf16", 1, 1)])
def test_selection(T, E, k, S, sigmoid, renorm, biased, masked, name, pad, shift):
    rng = np.random.default_rng([T, E, k, pad])
    x = _logits(rng, T, E, name)
    bias = torch.from_numpy(rng.normal(0, 0.1, E)).float().cuda() if biased else None
    mask = torch.from_numpy((rng.random(T) < 0.8).astype(np.uint8) * 7).cuda() if masked else None
    Call(x, k, S, sigmoid, renorm, bias, mask, scale=2.5 if sigmoid else 1.0, pad=pad, shift=shift).run().check()


@pytest.mark.parametrize("T,E,k,groups,top,best", [(50, 64, 6, 8, 3, 2), (50, 64, 6, 8, 3, 1), (300, 256, 8, 8, 4, 2), (40, 256, 2, 256, 2, 1), (40, 256, 8, 128, 5, 2),
                                                   (70, 60, 4, 6, 1, 2), (33, 30, 5, 3, 3, 2), (9, 7, 1, 7, 1, 1), (64, 96, 16, 2, 1, 2)])
@pytest.mark.parametrize("sigmoid,biased,name", [(True, True, "f32"), (False, False, "f32"), (True, False, "bf16"), (False, True, "bf16")])
def test_groups(T, E, k, groups, top, best, sigmoid, biased, name):
    rng = np.random.default_rng([T, E, groups, top])
    bias = torch.from_numpy(rng.normal(0, 0.1, E)).float().cuda() if biased else None
    Call(_logits(rng, T, E, name), k, 0, sigmoid, True, bias, None, groups, top, best, 2.0).run().check()


@pytest.mark.parametrize("E,top,k", [(256, 1, 16), (256, 2, 8), (256, 3, 6), (256, 5, 8), (256, 7, 16), (160, 3, 8), (160, 4, 1), (192, 4, 16), (192, 6, 8), (224, 2, 9)])
@pytest.mark.parametrize("sigmoid,biased,best,name", [(True, True, 2, "f32"), (False, False, 2, "f32"), (True, False, 1, "bf16"), (False, True, 1, "bf16")])
def test_groups_of_32(E, top, k, sigmoid, biased, best, name):
    rng = np.random.default_rng([E, top, k])
    x = _logits(rng, 90, E, name)
    x[20:40, 3::16] += 4.0                                              # most of the largest 16 apart
    x[40:60][torch.from_numpy(rng.random((20, E)) < 0.8).cuda()] = float("-inf")
    x[60:70, :32 * (E // 32 - 1)] = float("-inf")                       # one group left
    x[70, :] = float("-inf")
    x[71, 5] = 1.0
    x[72:80] = torch.from_numpy(rng.integers(0, 3, (8, E)) * 0.5).to(x)  # ties
    bias = torch.from_numpy(rng.normal(0, 0.1, E)).float().cuda() if biased else None
    Call(x, k, 0, sigmoid, True, bias, None, E // 32, top, best, 2.0).run().check()


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("groups,top,best", [(1, 1, 1), (8, 3, 2), (8, 3, 1)])
@pytest.mark.parametrize("E", [32, 64, 256])
def test_scores_that_fp32_does_not_tell_apart(sigmoid, groups, top, best, E):
    """Biases that bring every candidate of a row to the same sum but for roundings: the order is that of 64 bits."""
    rng = np.random.default_rng([E, groups])
    row = np.float32(rng.normal(0, 1.5, E))
    s = scores(row[None].astype(np.float64), sigmoid)[0]
    bias = torch.from_numpy((0.75 - s).astype(np.float32)).cuda()
    x = torch.from_numpy(np.repeat(row[None], 40, 0)).cuda()
    x[1::2] += torch.from_numpy(rng.normal(0, 1e-6, (20, E)).astype(np.float32)).cuda()
    Call(x, 8, 0, sigmoid, True, bias, None, groups, top, best).run().check()


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("biased", [False, True])
def test_ties_go_to_the_lower_index(sigmoid, biased):
    rng = np.random.default_rng(4)
    x = torch.from_numpy(rng.integers(0, 3, (100, 96)) * 0.5).float().cuda()
    x[0] = 0.25
    bias = torch.zeros(96, device="cuda") if biased else None
    for groups, top, best in ((1, 1, 1), (12, 4, 2), (12, 4, 1), (3, 2, 2)):
        Call(x, 6, 0, sigmoid, False, bias, None, groups, top, best).run().check()
        Call(x.bfloat16(), 6, 0, sigmoid, False, bias, None, groups, top, best).run().check()


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("E,groups,top,best", [(8, 1, 1, 1), (100, 1, 1, 1), (64, 4, 2, 1), (96, 12, 3, 1), (256, 8, 4, 2)])
def test_zeros_of_either_sign_tie(E, groups, top, best, name):
    rng = np.random.default_rng(E)
    x = torch.from_numpy(np.where(rng.random((60, E)) < 0.5, -0.0, 0.0)).to(dt(name)).cuda()
    x[20:40][torch.from_numpy(rng.random((20, E)) < 0.5).cuda()] = -1.0
    x[40:][torch.from_numpy(rng.random((20, E)) < 0.1).cuda()] = 2.0 ** -20
    for sigmoid in (False, True):
        for k in (1, 3, 6):
            Call(x, k, 0, sigmoid, True, None, None, groups, top, best).run().check()


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("groups,top,best", [(1, 1, 1), (4, 2, 2)])
@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_masked_experts(sigmoid, biased, groups, top, best, name):
    """Experts of -inf are never selected; rows that keep too few, or none, end in -1."""
    rng = np.random.default_rng(5)
    T, E, k = 80, 32, 5
    x = _logits(rng, T, E, name)
    for t in range(T):
        x[t, torch.from_numpy(rng.permutation(E)[:rng.integers(0, E + 1)]).cuda()] = float("-inf")
    x[3] = float("-inf")
    x[4, 1:] = float("-inf")
    bias = torch.from_numpy(rng.normal(0, 1, E)).float().cuda() if biased else None
    c = Call(x, k, 1, sigmoid, True, bias, None, groups, top, best).run().check()
    assert (c.outputs()[0][3] == -1).all() and (c.outputs()[1][3] == 0).all()


def test_all_rows_masked_and_no_rows():
    x = torch.full((70, 9), float("nan"), device="cuda")
    c = Call(x, 3, 2, mask=torch.zeros(70, dtype=torch.uint8, device="cuda")).run().check()
    assert (c.outputs()[4] == -1).all()
    Call(x[:0], 3, 2).run().check()


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("biased", [False, True])
def test_special_logits(sigmoid, biased):
    """NaN, and +inf under softmax: NaN weights and some experts, each once, none whose logit is NaN; rows beside them stay as they are."""
    rng = np.random.default_rng(6)
    T, E, k, inf = 40, 40, 6, float("inf")
    x = _logits(rng, T, E, "f32")
    x[1, 7], x[2, :] = float("nan"), float("nan")
    x[3, 5] = inf
    x[4, :8], x[5, 0] = inf, 3.4e38
    x[6] = torch.where(x[6] > 0, 3.4e38, -3.4e38)
    bias = torch.from_numpy(rng.normal(0, 0.1, E)).float().cuda() if biased else None
    c = Call(x, k, 0, sigmoid, True, bias, None, 4, 2, 2).run()
    torch.cuda.synchronize()
    i, w, counts, offsets, order, pos = c.outputs()
    bad = [1, 2] if sigmoid else [1, 2, 3, 4]
    good = [t for t in range(T) if t not in bad and not (sigmoid and t in (3, 4, 6)) and not (not sigmoid and t == 6)]
    idx, weight = select(f64(x)[good], k, sigmoid, True, None if bias is None else f64(bias), None, 4, 2, 2)
    assert np.array_equal(i[good], idx)
    assert (np.abs(w[good] - weight) <= STEPS * U32 * weight + 2.0 ** -120).all()
    xs = x.cpu().numpy()
    for t in range(T):
        got = i[t][i[t] >= 0]
        assert len(set(got)) == len(got) and (got < E).all() and not np.isnan(xs[t, got]).any()
        assert (len(got) == k) if t != 2 else len(got) == 0
        assert (np.isnan(w[t]) == ((i[t] >= 0) if t in bad else False)).all()
    for got, want in zip((counts, offsets, order, pos), pairs(i.astype(np.int64), None, E, 0)):
        assert np.array_equal(got, want)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("groups,top,best", [(1, 1, 1), (8, 3, 2)])
@pytest.mark.parametrize("E,of", [(256, 256), (256, 250), (200, 200), (64, 64), (16, 3)])
def test_biases_that_are_no_numbers(sigmoid, groups, top, best, E, of):
    """Selections from biases that a program let become NaN or infinite: some experts, each once, and their pairs."""
    rng = np.random.default_rng([E, of])
    x = _logits(rng, 70, E, "f32")
    for value in (float("nan"), float("inf"), -float("inf")):
        bias = torch.from_numpy(rng.normal(0, 0.1, E)).float().cuda()
        bias[torch.from_numpy(rng.permutation(E)[:of]).cuda()] = value
        c = Call(x, 3, 0, sigmoid, True, bias, None, groups, top, best).run()
        torch.cuda.synchronize()
        i, w, counts, offsets, order, pos = c.outputs()
        assert all(g.intact() for g in (c.X, c.idx, c.w, c.counts, c.offsets, c.order, c.pos, c.ws))
        assert ((i >= -1) & (i < E)).all()
        for t in range(70):
            got = i[t][i[t] >= 0]
            assert len(set(got)) == len(got)
        for got, want in zip((counts, offsets, order, pos), pairs(i.astype(np.int64), None, E, 0)):
            assert np.array_equal(got, want)


@pytest.mark.parametrize("outs", ["", "w", "c", "o", "f", "p", "wop"])
@pytest.mark.parametrize("T", [20, 500])
def test_optional_outputs(outs, T):
    rng = np.random.default_rng(8)
    x = _logits(rng, T, 24, "f32")
    full, part = Call(x, 3, 1).run().check(), Call(x, 3, 1, outs=outs).run()
    torch.cuda.synchronize()
    for n, a, b in zip("iwcofp", full.outputs(), part.outputs()):
        if n == "i" or n in outs:
            assert np.array_equal(a, b)
        else:
            assert (b.view(np.uint8) == 0xA5).all()


def test_as_the_fused_router():
    """The softmax selection of given logits is the one that the routing call makes from them."""
    T, C, E, k, S = 300, 256, 24, 4, 2
    g = torch.Generator(device="cuda").manual_seed(3)
    x, wr = torch.randn(T, C, generator=g, device="cuda").bfloat16(), (torch.randn(E, C, generator=g, device="cuda") / 16).bfloat16()
    i32 = lambda *s: torch.empty(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    shape = mira.MoEShape(C, 64, E, k, S, mira.MIRA_BF16)
    nb, stride = mira.mira_workspace_bytes(shape, T), mira.mira_packed_expert_bytes(C, 64)
    a = mira.MoEArgs(x=x, n_tokens=T, n_slots=1, w_router=wr, slot_table=i32(E + S).zero_(), slot_pool=torch.zeros(stride, dtype=torch.uint8, device="cuda"),
                     slot_stride=stride, out=torch.empty(T, C, device="cuda"), topk_idx=i32(T, k), topk_weight=torch.empty(T, k, device="cuda"),
                     logits=torch.empty(T, E, device="cuda"), expert_counts=i32(E + S), expert_offsets=i32(E + S + 1), pair_order=i32(T * (k + S)),
                     workspace=torch.empty(nb, dtype=torch.uint8, device="cuda"), workspace_bytes=nb)
    mira.mira_moe_route(shape, a)
    c = Call(a.logits, k, S, renorm=True).run().check()
    i, w, counts, offsets, order, pos = c.outputs()
    assert np.array_equal(i, a.topk_idx.cpu().numpy()) and np.array_equal(order, a.pair_order.cpu().numpy())
    assert np.array_equal(counts, a.expert_counts.cpu().numpy()) and np.array_equal(offsets, a.expert_offsets.cpu().numpy())
    assert np.allclose(w, a.topk_weight.cpu().numpy(), rtol=2 * STEPS * U32, atol=0)
    back = Guarded(1, T * (k + S), torch.int32)
    mira.mira_pair_positions(a.pair_order, T * (k + S), T * (k + S), back.v)
    torch.cuda.synchronize()
    assert back.intact() and np.array_equal(back.v[0].cpu().numpy(), pos)


def test_pair_positions_of_a_partial_order():
    order = torch.tensor([4, -1, 0, 9, 2, 12, 2 ** 31 - 1, 7], dtype=torch.int32, device="cuda")
    pos = Guarded(1, 10, torch.int32)
    mira.mira_pair_positions(order, 8, 10, pos.v)
    torch.cuda.synchronize()
    assert pos.intact() and pos.v[0].tolist() == [2, -1, 4, -1, 0, -1, -1, 7, -1, 3]
    mira.mira_pair_positions(None, 0, 10, pos.v)
    torch.cuda.synchronize()
    assert pos.v[0].tolist() == [-1] * 10


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (16, 8, 2), (300, 61, 4), (77, 64, 16), (130, 100, 3), (65, 256, 8), (2000, 12, 5),
                                   (33, 2, 2), (50, 3, 1), (65, 5, 4), (19, 129, 16), (40, 255, 1)])
@pytest.mark.parametrize("sigmoid,renorm,add,name,pad,shift", [(False, False, False, "f32", 0, 0), (False, True, True, "f32", 3, 1), (True, True, False, "bf16", 0, 0),
                                                               (True, False, True, "bf16", 5, 3), (False, False, True, "bf16", 1, 1), (True, True, True, "f32", 2, 0)])
def test_gradient(T, E, k, sigmoid, renorm, add, name, pad, shift):
    rng = np.random.default_rng([T, E, k, pad, 3])
    X = Guarded(T, E, dt(name), E + pad, shift).put(_logits(rng, T, E, name))
    idx = np.argsort(rng.random((T, E)), 1)[:, :k].astype(np.int32)
    idx[rng.random((T, k)) < 0.1] = -1
    idx[rng.random((T, k)) < 0.05] = E + 3
    idx[rng.random(T) < 0.1] = -1
    g = rng.normal(0, 1, (T, k)).astype(np.float32)
    gone = (idx < 0) | (idx >= E)
    X.v[torch.from_numpy(gone.all(1)).cuda()] = float("nan")
    I, G = (Guarded(T, k, t).put(torch.from_numpy(np.where(gone, np.float32("nan"), g) if t == torch.float32 else idx).cuda())
            for t in (torch.int32, torch.float32))
    A = Guarded(T, E, dt(name), E + 2 * pad, shift).put(torch.from_numpy(rng.normal(0, 1, (T, E))).cuda())
    D = Guarded(T, E, dt(name), E + 3 * pad, shift)
    scale = 2.5 if sigmoid else 1.0
    args = mira.RouteSelectGradArgs(logits=X.v, topk_idx=I.v, dweight=G.v, add=A.v if add else None, logits_dtype=code(name), n_tokens=T, n_experts=E, top_k=k,
                                    flags=(mira.MIRA_ROUTE_SIGMOID if sigmoid else 0) | (mira.MIRA_ROUTE_RENORM if renorm else 0), scale=scale, ld_logits=X.ld,
                                    ld_add=A.ld, ld_dlogits=D.ld, dlogits=D.v)
    mira.mira_route_select_grad(args)
    torch.cuda.synchronize()
    assert all(b.intact() for b in (X, I, G, A, D))
    with np.errstate(invalid="ignore"):
        want, mag = select_grad(np.where(np.isnan(f64(X.v)), 0.0, f64(X.v)), idx, g.astype(np.float64), sigmoid, renorm, scale)
    if add:
        want, mag = want + f64(A.v), mag + np.abs(f64(A.v))
    off = 2 * STEPS * U32 * mag
    assert (np.abs(f64(D.v) - want) <= off + unit(name) * (np.abs(want) + off) + 2.0 ** -120).all()
    first = D.v.clone()
    if add:
        args.dlogits, args.ld_dlogits = A.v, A.ld
        mira.mira_route_select_grad(args)
        torch.cuda.synchronize()
        assert torch.equal(A.v, first)
    else:
        args.dlogits, args.ld_dlogits = X.v, X.ld
        mira.mira_route_select_grad(args)
        torch.cuda.synchronize()
        assert torch.equal(X.v, first)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("E", [4, 100, 200])
def test_gradient_of_an_expert_selected_twice(sigmoid, renorm, E):
    """Each entry counts, whatever it selects."""
    rng = np.random.default_rng(E)
    x = _logits(rng, 40, E, "f32")
    idx = torch.from_numpy(rng.integers(0, 4, (40, 6)).astype(np.int32)).cuda()
    g, d = torch.randn(40, 6, device="cuda"), torch.empty(40, E, device="cuda")
    flags = (mira.MIRA_ROUTE_SIGMOID if sigmoid else 0) | (mira.MIRA_ROUTE_RENORM if renorm else 0)
    mira.mira_route_select_grad(mira.RouteSelectGradArgs(logits=x, topk_idx=idx, dweight=g, n_tokens=40, n_experts=E, top_k=6, flags=flags, dlogits=d))
    torch.cuda.synchronize()
    want, mag = select_grad(f64(x), idx.cpu().numpy(), f64(g), sigmoid, renorm, 1.0)
    assert (np.abs(f64(d) - want) <= 2 * STEPS * U32 * mag + 2.0 ** -120).all()


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_of_special_logits(sigmoid, renorm):
    T, E, inf = 6, 70, float("inf")
    x = torch.randn(T, E, device="cuda")
    idx = torch.tensor([[3, 9, 40]] * T, dtype=torch.int32, device="cuda")
    x[0, 50] = -inf        # masked expert, not selected
    x[1, 3] = -inf         # masked expert among the selected
    x[2, 50] = float("nan")
    x[3, 9] = float("nan")
    x[4] = -inf
    x[5, :] = torch.where(x[5] > 0, 80.0, -80.0)
    g = torch.randn(T, 3, device="cuda")
    d = torch.empty(T, E, device="cuda")
    flags = (mira.MIRA_ROUTE_SIGMOID if sigmoid else 0) | (mira.MIRA_ROUTE_RENORM if renorm else 0)
    mira.mira_route_select_grad(mira.RouteSelectGradArgs(logits=x, topk_idx=idx, dweight=g, n_tokens=T, n_experts=E, top_k=3, flags=flags, dlogits=d))
    torch.cuda.synchronize()
    got = f64(d)
    fine = [0, 1, 5] + ([2] if sigmoid else [])
    xs = f64(x)
    xs[2, 50] = 0.0 if sigmoid else xs[2, 50]
    want, mag = select_grad(xs[fine], idx.cpu().numpy()[fine], f64(g)[fine], sigmoid, renorm, 1.0)
    assert (np.abs(got[fine] - want) <= 2 * STEPS * U32 * mag + 2.0 ** -100).all()
    assert got[0, 50] == 0 and got[1, 3] == 0 and (got[4] == 0).all()
    if not sigmoid:
        assert np.isnan(got[2]).all() and np.isnan(got[3]).all()
    else:
        assert np.isnan(got[3, 9]) and np.isnan(got[3, [3, 40]]).all() == renorm
        assert (np.delete(got[3], [3, 9, 40]) == 0).all()


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_against_differences(sigmoid, renorm):
    """Central differences of the 64-bit weights of the experts that the forward call selected."""
    rng = np.random.default_rng(10)
    T, E, k, scale = 6, 20, 4, 1.7
    x = _logits(rng, T, E, "f32")
    c = Call(x, k, 0, sigmoid, renorm, torch.from_numpy(rng.normal(0, 0.3, E)).float().cuda(), None, 4, 2, 2, scale).run().check()
    g = torch.randn(T, k, device="cuda")
    d = torch.empty(T, E, device="cuda")
    mira.mira_route_select_grad(mira.RouteSelectGradArgs(logits=x, topk_idx=c.idx.v, dweight=g, n_tokens=T, n_experts=E, top_k=k, flags=c.args.flags,
                                                         scale=scale, dlogits=d))
    torch.cuda.synchronize()
    idx, xs, gs = c.idx.v.cpu().numpy(), f64(x), f64(g)

    def loss(v):
        s = np.take_along_axis(scores(v, sigmoid), idx.astype(np.int64), 1)
        return (gs * (s * scale / (s.sum(1, keepdims=True) + 1e-20) if renorm else s * scale)).sum()

    step = 1e-4   # off by step^2 / 6 times third derivatives (about 1) and 1e-16 / step
    for t, e in [(t, e) for t in range(T) for e in (int(idx[t, 0]), int(idx[t, 3]), (int(idx[t, 0]) + 1) % E)]:
        v = np.zeros_like(xs)
        v[t, e] = step
        assert abs((loss(xs + v) - loss(xs - v)) / (2 * step) - float(d[t, e])) < 1e-6


def test_far_rows():
    ld, T, E, k = 1 << 27, 40, 70, 3
    rng = np.random.default_rng(12)
    x = _logits(rng, T, E, "f32")
    far = torch.empty(T * ld, device="cuda").view(T, ld)
    far[:, :E] = x
    a = Call(x, k, 1).run().check()
    b = Call(x, k, 1)
    b.args.logits, b.args.ld_logits = far, ld
    b.run().check()
    g, d = torch.randn(T, k, device="cuda"), torch.empty(T, E, device="cuda")
    base = dict(topk_idx=a.idx.v, dweight=g, n_tokens=T, n_experts=E, top_k=k)
    mira.mira_route_select_grad(mira.RouteSelectGradArgs(logits=x, dlogits=d, **base))
    mira.mira_route_select_grad(mira.RouteSelectGradArgs(logits=far, ld_logits=ld, dlogits=far[:, 512:], ld_dlogits=ld, **base))
    torch.cuda.synchronize()
    assert torch.equal(far[:, 512:512 + E], d)
    del far
    torch.cuda.empty_cache()


@pytest.mark.parametrize("T,E,k", [(131072, 32, 2), (70000, 8, 1), (20000, 200, 8)])
def test_many_tokens(T, E, k):
    """Every chunking of long batches: the order against a stable sort."""
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, E, generator=g, device="cuda")
    mask = (torch.rand(T, generator=g, device="cuda") < 0.9).to(torch.uint8)
    c = Call(x, k, 1, renorm=True, mask=mask).run()
    torch.cuda.synchronize()
    idx = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k].masked_fill(mask[:, None] == 0, -1)
    assert torch.equal(c.idx.v.long(), idx)
    group = torch.cat([idx.reshape(-1), torch.full((T,), E, device="cuda").masked_fill(mask == 0, -1)])
    group = torch.where(group < 0, E + 1, group)
    order = torch.sort(group, stable=True).indices
    n = int((group <= E).sum())
    assert torch.equal(c.order.v[0, :n].long(), order[:n]) and (c.order.v[0, n:] == -1).all()
    pos = torch.empty_like(order)
    pos[order] = torch.arange(len(order), device="cuda")
    assert torch.equal(c.pos.v[0].long(), torch.where(pos < n, pos, -1))
    assert torch.equal(c.counts.v[0].long(), torch.bincount(group, minlength=E + 2)[:E + 1])
    assert torch.equal(c.offsets.v[0, 1:].long(), c.counts.v[0].long().cumsum(0))
    assert all(b.intact() for b in (c.X, c.idx, c.w, c.counts, c.offsets, c.order, c.pos, c.ws))


def _few_experts(E, k, name, seed):
    """Rows with all that a row may have: usual ones, ties, experts of -inf, rows of them, neighbours that fp32 does not tell apart, NaN, infinities."""
    rng = np.random.default_rng([E, k, seed])
    T = 8800
    x = _logits(rng, T, E, name)
    x[1000:2000] = torch.from_numpy(rng.integers(-1, 2, (1000, E)) * 0.5).to(x)
    x[2000:2400][torch.from_numpy(rng.random((400, E)) < 0.5).cuda()] = float("-inf")
    x[2400:2410] = float("-inf")
    x[2500:2600] = torch.from_numpy(rng.normal(0, 1, (100, 1)) + rng.normal(0, 1e-6, (100, E))).to(x)
    x[2600:2700] *= 40
    x[2700:2800] = torch.where(torch.from_numpy(rng.random((100, E)) < 0.5).cuda(), -0.0, 0.0).to(x)
    return rng, x


@pytest.mark.parametrize("E,k", [(1, 1), (2, 2), (3, 1), (7, 4), (8, 2), (8, 4), (9, 3), (15, 4), (16, 1), (16, 4), (8, 5), (16, 8), (17, 1), (17, 8), (33, 5), (61, 7), (63, 8), (64, 6),
                                 (64, 8)])
@pytest.mark.parametrize("sigmoid,renorm,biased,name,pad,shift", [(False, True, False, "f32", 0, 0), (True, True, True, "bf16", 3, 1),
                                                                  (False, False, True, "f32", 1, 1), (True, False, False, "bf16", 0, 0)])
def test_long_batches_of_few_experts(E, k, sigmoid, renorm, biased, name, pad, shift):
    rng, x = _few_experts(E, k, name, 0)
    T = len(x)
    bias = torch.from_numpy(rng.normal(0, 0.1, E)).float().cuda() if biased else None
    mask = torch.from_numpy((rng.random(T) < 0.9).astype(np.uint8)).cuda() if shift else None
    c = Call(x, k, 2 if E < 9 else 0, sigmoid, renorm, bias, mask, scale=2.5, pad=pad, shift=shift).run()
    # fp32 holds v - max to half a step, which is that much of exp(v - max) relatively, and no score below 2^-126; both count
    # in rows of logits this far apart (half a step of -65 is 64 half steps of 1)
    xs, i = f64(c.X.v), c.outputs()[0]
    top, of = xs.max(1, keepdims=True), np.take_along_axis(xs, np.maximum(i, 0), 1)
    s = np.where(i >= 0, np.take_along_axis(scores(xs, sigmoid), np.maximum(i, 0), 1), 0.0)
    share = 2.5 / (s.sum(1, keepdims=True) + TINY) if renorm else 2.5
    with np.errstate(invalid="ignore"):
        apart = np.where((i >= 0) & ~np.isneginf(top), top - of, 0.0)
    c.check(extra=(0.0 if sigmoid else U32 * apart * s * share) + 2.0 ** -126 * share)
    # a batch that is not long: the same bits
    d = Call(x[:4400], k, 0, sigmoid, renorm, bias, None if mask is None else mask[:4400], scale=2.5, pad=pad, shift=shift).run()
    torch.cuda.synchronize()
    assert torch.equal(c.idx.v[:4400], d.idx.v) and torch.equal(c.w.v[:4400], d.w.v)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("E,k", [(8, 3), (40, 6)])
def test_long_batches_special_logits(sigmoid, biased, E, k):
    """NaN and infinities in a long batch of few experts: the selection and weights of a shorter one."""
    rng, x = _few_experts(E, k, "f32", 1)
    x[torch.from_numpy(rng.random(tuple(x.shape)) < 0.02).cuda()] = float("nan")
    x[torch.from_numpy(rng.random(tuple(x.shape)) < 0.02).cuda()] = float("inf")
    bias = torch.from_numpy(rng.normal(0, 0.1, E)).float().cuda() if biased else None
    c, d = Call(x, k, 0, sigmoid, True, bias).run(), Call(x[:4400], k, 0, sigmoid, True, bias).run()
    torch.cuda.synchronize()
    assert torch.equal(c.idx.v[:4400], d.idx.v) and torch.equal(c.w.v[:4400].view(torch.int32), d.w.v.view(torch.int32))
    i = c.outputs()[0]
    xs = x.cpu().numpy()
    for t in range(len(xs)):
        got = i[t][i[t] >= 0]
        assert len(set(got)) == len(got) and not np.isnan(xs[t, got]).any()
    for got, want in zip(c.outputs()[2:], pairs(i.astype(np.int64), None, E, 0)):
        assert np.array_equal(got, want)
    assert all(b.intact() for b in (c.X, c.idx, c.w, c.counts, c.offsets, c.order, c.pos, c.ws))


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("E,k", [(16, 4), (64, 8)])
def test_long_batches_scores_that_fp32_does_not_tell_apart(sigmoid, E, k):
    rng = np.random.default_rng(14)
    row = np.float32(rng.normal(0, 1.5, E))
    bias = torch.from_numpy((0.75 - scores(row[None].astype(np.float64), sigmoid)[0]).astype(np.float32)).cuda()
    x = torch.from_numpy(np.repeat(row[None], 8300, 0)).cuda()
    x[1::2] += torch.from_numpy(rng.normal(0, 1e-6, (4150, E)).astype(np.float32)).cuda()
    Call(x, k, 0, sigmoid, True, bias).run().check()


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("E", [6, 70, 130, 200])
@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_gradient_of_masked_experts_counts_for_nothing(sigmoid, renorm, E, name):
    """Entries of experts of -inf leave the row what it is without them, whatever arrives at them."""
    rng = np.random.default_rng([E, 5])
    T, k = 64, 3
    x = _logits(rng, T, E, name)
    idx = np.argsort(rng.random((T, E)), 1)[:, :k].astype(np.int32)
    g = rng.normal(0, 1, (T, k)).astype(np.float32)
    gone = rng.random((T, k)) < 0.4
    gone[:8] = True                      # all of the row's entries
    for t, j in zip(*np.nonzero(gone)):
        x[t, int(idx[t, j])] = float("-inf")
    g[gone] = rng.choice(np.float32([np.nan, np.inf, -np.inf, 3e38, 1.0]), gone.sum())
    free = [int(next(e for e in range(E) if e not in idx[t])) for t in range(8)]
    for t in range(4):
        x[t, free[t]] = float("nan") if t % 2 else float("inf")   # a row without other entries: 0 all the same
    add, d = torch.from_numpy(rng.normal(0, 1, (T, E))).to(x), torch.empty_like(x)
    flags = (mira.MIRA_ROUTE_SIGMOID if sigmoid else 0) | (mira.MIRA_ROUTE_RENORM if renorm else 0)
    base = dict(logits=x, topk_idx=torch.from_numpy(idx).cuda(), dweight=torch.from_numpy(g).cuda(), logits_dtype=code(name), n_tokens=T, n_experts=E, top_k=k,
                flags=flags, dlogits=d)
    without = np.where(gone, -1, idx)
    xs = f64(x)
    xs[:4] = 0.0                         # (no entry: no logit of theirs counts)
    want, mag = select_grad(xs, without, np.where(gone, 0.0, g.astype(np.float64)), sigmoid, renorm, 1.0)
    for a in (None, add):
        mira.mira_route_select_grad(mira.RouteSelectGradArgs(add=a, **base))
        torch.cuda.synchronize()
        w, m = (want, mag) if a is None else (want + f64(add), mag + np.abs(f64(add)))
        off = 2 * STEPS * U32 * m
        assert (np.abs(f64(d) - w) <= off + unit(name) * (np.abs(w) + off) + 2.0 ** -120).all()


@pytest.mark.parametrize("T,E,k,groups,top,best", [(70, 8, 2, 1, 1, 1), (70, 40, 6, 1, 1, 1), (70, 100, 8, 1, 1, 1), (70, 256, 8, 1, 1, 1), (70, 256, 8, 8, 4, 2),
                                                   (70, 60, 4, 6, 2, 2), (70, 64, 4, 8, 3, 1), (8300, 8, 2, 1, 1, 1), (8300, 16, 4, 1, 1, 1), (8300, 40, 6, 1, 1, 1)])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("biases", ["one at -1e9", "one at 1e4", "all at 1000", "one at 3e38", "all at 3e38", "one at -3.4e38", "both ends"])
def test_biases_far_apart(T, E, k, groups, top, best, sigmoid, biases):
    """Biases beside which a score is little or nothing, such as switch an expert off or on: the order is that of 64 bits."""
    rng = np.random.default_rng([T, E, len(biases)])
    b = np.float32(rng.normal(0, 0.1, E))
    at = int(rng.integers(E))
    if biases == "both ends":
        b[at], b[(at + 1) % E] = 3.4e38, -3.4e38
    elif biases.startswith("one"):
        b[at] = np.float32(biases.split()[-1])
    else:
        b = np.float32(float(biases.split()[-1]) + (b if biases.endswith("1000") else 0 * b))
    Call(_logits(rng, T, E, "f32"), k, 0, sigmoid, True, torch.from_numpy(b).cuda(), None, groups, top, best, 2.5).run().check()


@pytest.mark.parametrize("T,E,k", [(131072, 255, 8), (131072, 24, 2), (60000, 100, 8)])
def test_more_chunks_and_pairs_than_one_step_takes(T, E, k):
    """Counts of chunks over several steps, with a carry and without a launch for them; more pairs in a chunk than its threads keep."""
    test_many_tokens(T, E, k)


@pytest.mark.parametrize("T,E,k,S", [(64, 100, 16, 17), (128, 64, 16, 3), (60, 256, 16, 0), (64, 200, 16, 56), (500, 64, 16, 60)])
def test_many_pairs_of_few_tokens(T, E, k, S):
    rng = np.random.default_rng([T, E, k, S])
    mask = torch.from_numpy((rng.random(T) < 0.8).astype(np.uint8)).cuda()
    Call(_logits(rng, T, E, "f32"), k, S, True, True, None, mask).run().check()
