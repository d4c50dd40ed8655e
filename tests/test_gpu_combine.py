"""The combine of the pairs' rows and its gradients against 64 bits: types, odd
sizes, strides, shared pairs, positions that are missing or out of range, 8-bit
rows, rows that no pair has."""
import numpy as np
import pytest
import torch

import paper_2609_38090_amd as mira
from layer_reference import U32, Guarded, code, dt, e4m3_close, f64, unit
from ops_reference import TABLE

pytestmark = pytest.mark.gpu
SIZES = [(1, 2, 0, 4096), (1, 1, 0, 1), (16, 6, 2, 2048), (5, 3, 1, 511), (7, 2, 0, 513), (9, 16, 3, 1025), (301, 4, 0, 127), (40, 8, 2, 2001),
         (3, 2, 1, 20011), (4500, 1, 0, 64), (6, 7, 0, 1500)]


def _pairs(rng, T, k, S, extra=5, missing=0.1):
    """Positions of the pairs among y_rows rows, some of them missing (-1, or out of range)."""
    n = T * (k + S)
    pos = rng.permutation(n + extra)[:n].astype(np.int32)
    if missing:
        gone = rng.random(n) < missing
        pos[gone] = rng.choice([-1, -7, n + extra, 2 ** 31 - 1], gone.sum())
    return pos, n + extra


def _by_token(pos, T, k, S, y_rows):
    at = np.concatenate([pos[:T * k].reshape(T, k), pos[T * k:].reshape(S, T).T], 1).astype(np.int64)
    return np.where((at >= 0) & (at < y_rows), at, -1)


@pytest.mark.parametrize("T,k,S,cols", SIZES)
@pytest.mark.parametrize("y,o,weights,res,pad,shift,missing", [("bf16", "bf16", True, True, 0, 0, 0.0), ("f32", "f32", True, False, 0, 0, 0.2),
                                                               ("f32", "bf16", False, True, 3, 1, 0.1), ("bf16", "f32", True, True, 5, 3, 0.1)])
def test_forward(T, k, S, cols, y, o, weights, res, pad, shift, missing):
    rng = np.random.default_rng([T, k, cols, pad])
    pos, rows = _pairs(rng, T, k, S, missing=missing)
    Y = Guarded(rows, cols, dt(y), cols + pad, shift).put(torch.from_numpy(rng.normal(0, 1, (rows, cols))).cuda())
    W = Guarded(T, k, torch.float32).put(torch.from_numpy(rng.random((T, k))).float().cuda())
    P = Guarded(1, T * (k + S), torch.int32).put(torch.from_numpy(pos).cuda())
    R = Guarded(T, cols, dt(o), cols + pad, shift).put(torch.from_numpy(rng.normal(0, 1, (T, cols))).cuda())
    O = Guarded(T, cols, dt(o), cols + 2 * pad, shift)
    args = mira.CombineArgs(y=Y.v, topk_weight=W.v if weights else None, pair_pos=P.v, residual=R.v if res else None, n_tokens=T, top_k=k, n_shared=S,
                            cols=cols, y_rows=rows, y_dtype=code(y), out_dtype=code(o), ldy=Y.ld, ld_res=R.ld, out=O.v, ld_out=O.ld)
    mira.mira_combine(args)
    torch.cuda.synchronize()
    assert all(g.intact() for g in (Y, W, P, R, O))
    at = _by_token(pos, T, k, S, rows)
    w = np.concatenate([f64(W.v) if weights else np.ones((T, k)), np.ones((T, S))], 1) * (at >= 0)
    terms = f64(Y.v)[at] * w[:, :, None]
    want, mag = terms.sum(1), np.abs(terms).sum(1)
    if res:
        want, mag = want + f64(R.v), mag + np.abs(f64(R.v))
    off = (k + S + 1) * U32 * mag
    assert (np.abs(f64(O.v) - want) <= off + unit(o) * (np.abs(want) + off)).all()
    if res:
        first = O.v.clone()
        args.out, args.ld_out = R.v, R.ld
        mira.mira_combine(args)
        torch.cuda.synchronize()
        assert torch.equal(R.v, first)


@pytest.mark.parametrize("T,k,S,cols", SIZES)
@pytest.mark.parametrize("y,o,outs,weights,pad,shift,missing", [
    ("bf16", "bf16", "qw", True, 0, 0, 0.0), ("f32", "f32", "dyw", True, 0, 0, 0.2), ("f32", "bf16", "dyqw", False, 3, 1, 0.1),
    ("bf16", "f32", "dyq", True, 5, 3, 0.1), ("bf16", "bf16", "w", True, 0, 0, 0.1)])
def test_gradient(T, k, S, cols, y, o, outs, weights, pad, shift, missing):
    rng = np.random.default_rng([T, k, cols, pad, 1])
    pos, rows = _pairs(rng, T, k, S, missing=missing)
    Y = Guarded(rows, cols, dt(y), cols + pad, shift).put(torch.from_numpy(rng.normal(0, 1, (rows, cols))).cuda())
    D = Guarded(T, cols, dt(o), cols + 2 * pad, shift).put(torch.from_numpy(rng.normal(0, 1, (T, cols))).cuda())
    W = Guarded(T, k, torch.float32).put(torch.from_numpy(rng.normal(0, 1, (T, k))).float().cuda())
    P = Guarded(1, T * (k + S), torch.int32).put(torch.from_numpy(pos).cuda())
    c16, nb = -(-cols // 16) * 16, -(-cols // 128)
    DY, DW = Guarded(rows, cols, dt(y), cols + pad, shift), Guarded(T, k, torch.float32)
    Q, C = Guarded(rows, c16, torch.uint8, c16 + 16 * (pad % 2)), Guarded(rows, nb, torch.float32, nb + pad)
    has = {n: n in outs for n in ("dy", "q", "w")}
    args = mira.CombineGradArgs(dout=D.v, y=Y.v if has["w"] else None, topk_weight=W.v if weights else None, pair_pos=P.v, n_tokens=T, top_k=k, n_shared=S,
                                cols=cols, y_rows=rows, y_dtype=code(y), out_dtype=code(o), q_eps=1e-8, ld_dout=D.ld, ldy=Y.ld,
                                dy=DY.v if has["dy"] else None, ld_dy=DY.ld, q=Q.v if has["q"] else None, ldq=Q.ld, scale=C.v if has["q"] else None,
                                ld_scale=C.ld, dweight=DW.v if has["w"] else None)
    before = DY.v.clone(), Q.v.clone(), C.v.clone()
    mira.mira_combine_grad(args)
    torch.cuda.synchronize()
    assert all(g.intact() for g in (Y, D, W, P, DY, DW, Q, C))
    at, d = _by_token(pos, T, k, S, rows), f64(D.v)
    w = np.concatenate([f64(W.v) if weights else np.ones((T, k)), np.ones((T, S))], 1)
    used = np.zeros(rows, bool)
    want = np.zeros((rows, cols))
    for j in range(k + S):
        on = at[:, j] >= 0
        want[at[on, j]] = w[on, j][:, None] * d[on]
        used[at[on, j]] = True
    u = torch.from_numpy(used).cuda()
    if has["dy"]:
        assert (np.abs(f64(DY.v)[used] - want[used]) <= (U32 + unit(y)) * np.abs(want[used]) + 1e-38).all()
        assert torch.equal(DY.v[~u].view(torch.uint8), before[0][~u].view(torch.uint8))
    if has["q"]:
        assert (Q.v[u][:, cols:] == 0).all()
        assert e4m3_close(Q.v[u][:, :cols].cpu().numpy(), C.v[u].cpu().numpy(), want[used], TABLE, U32 * np.abs(want[used])).all()
        assert torch.equal(Q.v[~u], before[1][~u]) and torch.equal(C.v[~u].view(torch.int32), before[2][~u].view(torch.int32))
        if has["dy"] and y == "f32":   # byte for byte the quantizer's of fp32 rows
            q2, s2 = torch.empty(rows, c16, dtype=torch.uint8, device="cuda"), torch.empty(rows, nb, device="cuda")
            mira.mira_fp8_quantize(mira.Fp8QuantArgs(x=DY.v, x_dtype=mira.MIRA_F32, rows=rows, cols=cols, eps=1e-8, ldx=DY.ld, q=q2, scale=s2))
            torch.cuda.synchronize()
            assert torch.equal(q2[u], Q.v[u]) and torch.equal(s2[u], C.v[u])
    if has["w"]:
        prod = d[:, None, :] * f64(Y.v)[at[:, :k]] * (at[:, :k] >= 0)[:, :, None]
        # a thread's products one after another, the lanes' and the waves'
        steps = 8 * -(-cols // 2048) + 12
        assert (np.abs(f64(DW.v) - prod.sum(2)) <= steps * U32 * np.abs(prod).sum(2)).all()
    if has["dy"] and has["w"]:        # over y
        first = DY.v.clone(), DW.v.clone()
        args.dy, args.ld_dy = Y.v, Y.ld
        mira.mira_combine_grad(args)
        torch.cuda.synchronize()
        assert torch.equal(Y.v[u], first[0][u]) and torch.equal(DW.v, first[1])


def test_no_rows():
    """Without a row of y every pair is missing."""
    T, k, cols = 3, 2, 70
    pos = torch.zeros(T * k, dtype=torch.int32, device="cuda")
    out, res, dw = torch.empty(T, cols, device="cuda"), torch.randn(T, cols, device="cuda"), torch.full((T, k), 4.0, device="cuda")
    mira.mira_combine(mira.CombineArgs(pair_pos=pos, residual=res, n_tokens=T, top_k=k, cols=cols, y_rows=0, y_dtype=0, out_dtype=0, out=out))
    mira.mira_combine_grad(mira.CombineGradArgs(dout=res, pair_pos=pos, n_tokens=T, top_k=k, cols=cols, y_rows=0, y_dtype=0, out_dtype=0, dweight=dw))
    torch.cuda.synchronize()
    assert torch.equal(out, res) and (dw == 0).all()


def test_non_finite_rows_stay_their_own():
    """NaN in a row that no pair has does not spread, nor does a weight of a missing pair."""
    T, k, cols = 4, 2, 300
    y = torch.randn(T * k + 1, cols, device="cuda")
    y[3] = float("nan")
    pos = torch.tensor([0, 1, 2, -1, 4, 5, 6, 7], dtype=torch.int32, device="cuda")
    w = torch.rand(T, k, device="cuda")
    w[1, 1] = float("inf")
    out, dw = torch.empty(T, cols, device="cuda"), torch.empty(T, k, device="cuda")
    mira.mira_combine(mira.CombineArgs(y=y, topk_weight=w, pair_pos=pos, n_tokens=T, top_k=k, cols=cols, y_rows=T * k + 1, y_dtype=0, out_dtype=0, out=out))
    mira.mira_combine_grad(mira.CombineGradArgs(dout=out, y=y, topk_weight=w, pair_pos=pos, n_tokens=T, top_k=k, cols=cols, y_rows=T * k + 1, y_dtype=0,
                                                out_dtype=0, dweight=dw))
    torch.cuda.synchronize()
    assert torch.isfinite(out).all() and torch.isfinite(dw).all() and float(dw[1, 1]) == 0


def test_gradient_against_differences():
    T, k, S, cols = 3, 2, 1, 19
    rng = np.random.default_rng(3)
    pos, rows = _pairs(rng, T, k, S, missing=0.0)
    y, w, g = rng.normal(0, 1, (rows, cols)), rng.random((T, k)), rng.normal(0, 1, (T, cols))
    y, w, g = (v.astype(np.float32) for v in (y, w, g))
    dy, dw = torch.zeros(rows, cols, device="cuda"), torch.empty(T, k, device="cuda")
    t = [torch.from_numpy(v).cuda() for v in (g, y, w, pos)]
    mira.mira_combine_grad(mira.CombineGradArgs(dout=t[0], y=t[1], topk_weight=t[2], pair_pos=t[3], n_tokens=T, top_k=k, n_shared=S, cols=cols, y_rows=rows,
                                                y_dtype=0, out_dtype=0, dy=dy, dweight=dw))
    torch.cuda.synchronize()
    y, w, g = (v.astype(np.float64) for v in (y, w, g))
    at = _by_token(pos, T, k, S, rows)

    def loss(y, w):
        return (g * (y[at] * np.concatenate([w, np.ones((T, S))], 1)[:, :, None]).sum(1)).sum()

    step = 1e-4   # the loss is linear in each: differences are off by roundings alone
    for r, c in [(0, 0), (int(at[1, 2]), 3), (int(at[2, 0]), 18), (int(at[0, 1]), 7)]:
        d = np.zeros_like(y)
        d[r, c] = step
        assert abs((loss(y + d, w) - loss(y - d, w)) / (2 * step) - float(dy[r, c])) < 1e-6
    for i in range(T):
        d = np.zeros_like(w)
        d[i, i % k] = step
        assert abs((loss(y, w + d) - loss(y, w - d)) / (2 * step) - float(dw[i, i % k])) < 1e-5


def test_far_rows():
    ld, T, k, cols = 1 << 27, 8, 2, 300
    rng = np.random.default_rng(9)
    pos, rows = _pairs(rng, T, k, 0, extra=4, missing=0.0)
    y, w, p = torch.from_numpy(rng.normal(0, 1, (rows, cols))).cuda().bfloat16(), torch.rand(T, k, device="cuda"), torch.from_numpy(pos).cuda()
    far = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld)
    far[:, :cols] = y
    out, out2 = (torch.empty(T, cols, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    base = dict(topk_weight=w, pair_pos=p, n_tokens=T, top_k=k, cols=cols, y_rows=rows)
    mira.mira_combine(mira.CombineArgs(y=y, out=out, **base))
    mira.mira_combine(mira.CombineArgs(y=far, ldy=ld, out=out2, **base))
    dy, dw, dw2 = torch.zeros_like(y), torch.empty_like(w), torch.empty_like(w)
    far[:, 512:512 + cols] = 0
    mira.mira_combine_grad(mira.CombineGradArgs(dout=out, y=y, dy=dy, dweight=dw, **base))
    mira.mira_combine_grad(mira.CombineGradArgs(dout=out, y=far, ldy=ld, dy=far[:, 512:], ld_dy=ld, dweight=dw2, **base))
    torch.cuda.synchronize()
    assert torch.equal(out, out2) and torch.equal(dw, dw2) and torch.equal(far[:, 512:512 + cols], dy)
    del far
    torch.cuda.empty_cache()


@pytest.mark.parametrize("T,k,S,cols", [(5, 16, 49, 130), (3, 8, 60, 700), (2, 1, 64, 33), (4, 5, 75, 130), (1, 16, 256, 2100), (3, 16, 48, 130)])
@pytest.mark.parametrize("y,o,pad,shift", [("bf16", "bf16", 0, 0), ("f32", "bf16", 3, 1), ("f32", "f32", 5, 3)])
def test_more_pairs_than_lanes(T, k, S, cols, y, o, pad, shift):
    """Tokens of 64 and more pairs, missing ones among all of them."""
    test_forward(T, k, S, cols, y, o, True, True, pad, shift, 0.3)
    test_gradient(T, k, S, cols, y, o, "dyqw", True, pad, shift, 0.3)
