"""The norm with the residual's addition and its 8-bit output, and its gradient,
against 64 bits: types, odd sizes, strides, alignments, rows that registers do not
hold, values at the ends of the range, buffers in each other's place, streams."""
import numpy as np
import pytest
import torch

import paper_2609_38090_amd as mira
from layer_reference import U32, Guarded, code, dt, e4m3_close, f64, norm, norm_grad, unit
from ops_reference import TABLE

pytestmark = pytest.mark.gpu
EPS, Q_EPS = 1e-6, 1e-8

# one row to many; a wave's rows, and those of 128 to 1024 threads, at and beside their ends; rows read twice
SIZES = [(1, 1), (3, 7), (1, 4096), (5, 512), (5, 513), (9, 1024), (9, 1025), (301, 2001), (4, 2048), (3, 4097), (2, 8192), (3, 8193),
         (2, 16384), (3, 16385), (2, 24577), (2050, 64), (1100, 700)]
# the longest chain of additions in a thread, the lanes' six and the waves' sixteen, then r and the products
CHAIN = {c: 8 * -(-c // 8192) + 8 + 22 for _, c in SIZES}


def _rows(rng, rows, cols):
    x = rng.normal(0, 1, (rows, cols)) * np.exp(rng.normal(0, 1, (rows, 1)))
    x[:, rng.integers(0, cols, max(1, cols // 200))] *= 20
    return torch.from_numpy(x).float().cuda()


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("x,w,y,res,pad,shift", [("bf16", "bf16", "bf16", True, 0, 0), ("f32", "f32", "f32", False, 0, 0),
                                                 ("bf16", "f32", "f32", True, 3, 1), ("f32", "bf16", "bf16", True, 5, 3)])
def test_forward(rows, cols, x, w, y, res, pad, shift):
    rng = np.random.default_rng([rows, cols, pad])
    X = Guarded(rows, cols, dt(x), cols + pad, shift).put(_rows(rng, rows, cols))
    R = Guarded(rows, cols, dt(x), cols + 2 * pad, shift).put(_rows(rng, rows, cols))
    W = Guarded(1, cols, dt(w), None, shift).put(1 + 0.2 * torch.from_numpy(rng.normal(0, 1, (1, cols))).float().cuda())
    S, Y = Guarded(rows, cols, dt(x), cols + pad, shift), Guarded(rows, cols, dt(y), cols + 3 * pad, shift)
    c16, nb = -(-cols // 16) * 16, -(-cols // 128)
    Q, C = Guarded(rows, c16, torch.uint8, c16 + 16 * (pad % 2)), Guarded(rows, nb, torch.float32, nb + pad)
    args = mira.RmsNormArgs(x=X.v, residual=R.v if res else None, weight=W.v, x_dtype=code(x), w_dtype=code(w), y_dtype=code(y), rows=rows,
                            cols=cols, eps=EPS, q_eps=Q_EPS, ldx=X.ld, ld_res=R.ld, sum=S.v, ld_sum=S.ld, y=Y.v, ldy=Y.ld, q=Q.v, ldq=Q.ld,
                            scale=C.v, ld_scale=C.ld)
    mira.mira_rmsnorm(args)
    torch.cuda.synchronize()
    assert all(g.intact() for g in (X, R, W, S, Y, Q, C))
    h = X.v + R.v if res else X.v          # one rounding of an exact sum of two (bf16 through fp32 is the same rounding)
    assert torch.equal(S.v, h)
    want, _ = norm(f64(h), f64(W.v), EPS)
    off = CHAIN[cols] * U32 * np.abs(want)
    assert (np.abs(f64(Y.v) - want) <= off + unit(y) * (np.abs(want) + off) + 1e-38).all()
    q, scale = Q.v.cpu().numpy(), C.v.cpu().numpy()
    assert (q[:, cols:] == 0).all()
    assert e4m3_close(q[:, :cols], scale, want, TABLE, off).all()
    # ... and byte for byte the quantizer's of y in fp32
    y32 = torch.empty(rows, cols, device="cuda")
    mira.mira_rmsnorm(mira.RmsNormArgs(x=S.v, weight=W.v, x_dtype=code(x), w_dtype=code(w), y_dtype=mira.MIRA_F32, rows=rows, cols=cols, eps=EPS,
                                       ldx=S.ld, y=y32))
    q2, s2 = torch.empty(rows, c16, dtype=torch.uint8, device="cuda"), torch.empty(rows, nb, device="cuda")
    mira.mira_fp8_quantize(mira.Fp8QuantArgs(x=y32, x_dtype=mira.MIRA_F32, rows=rows, cols=cols, eps=Q_EPS, q=q2, scale=s2))
    torch.cuda.synchronize()
    assert torch.equal(q2, Q.v) and torch.equal(s2, C.v)
    assert torch.equal(Y.v, y32.to(dt(y)))  # a call on the sum gives the same bits


@pytest.mark.parametrize("rows,cols", [(7, 300), (5, 4096), (3, 20000)])
@pytest.mark.parametrize("over", ["x", "residual"])
def test_sum_in_place(rows, cols, over):
    rng = np.random.default_rng(cols)
    x, r = _rows(rng, rows, cols).bfloat16(), _rows(rng, rows, cols).bfloat16()
    w = torch.ones(cols, dtype=torch.bfloat16, device="cuda")
    y, y2 = torch.empty_like(x), torch.empty_like(x)
    h = x + r
    mira.mira_rmsnorm(mira.RmsNormArgs(x=h, weight=w, rows=rows, cols=cols, y=y2))
    mira.mira_rmsnorm(mira.RmsNormArgs(x=x, residual=r, weight=w, rows=rows, cols=cols, sum=x if over == "x" else r, y=y))
    torch.cuda.synchronize()
    assert torch.equal(x if over == "x" else r, h) and torch.equal(y, y2)


@pytest.mark.parametrize("cols", [100, 4096, 9000, 20000])
def test_ends_of_the_range(cols):
    """Zeros, values whose squares pass fp32's range (and the largest there are), tiny ones, NaN and infinities."""
    rng = np.random.default_rng(cols)
    x = _rows(rng, 7, cols)
    x[0] = 0.0
    x[1] *= 1e30
    x[2] = torch.where(x[2] > 0, 3.4e38, -3.4e38)
    x[3] *= 1e-18
    x[4, cols // 2] = float("nan")
    x[5, cols - 1] = float("-inf")
    w = torch.ones(cols, device="cuda")
    y, q, s = torch.empty_like(x), torch.empty(7, -(-cols // 16) * 16, dtype=torch.uint8, device="cuda"), torch.empty(7, -(-cols // 128), device="cuda")
    mira.mira_rmsnorm(mira.RmsNormArgs(x=x, weight=w, x_dtype=0, w_dtype=0, y_dtype=0, rows=7, cols=cols, eps=EPS, y=y, q=q, scale=s))
    dy, dx = torch.from_numpy(rng.normal(0, 1, (7, cols))).float().cuda(), torch.empty_like(x)
    dw, nb = torch.empty(cols, device="cuda"), mira.mira_rmsnorm_grad_workspace_bytes(7, cols)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    mira.mira_rmsnorm_grad(mira.RmsNormGradArgs(dy=dy, h=x, weight=w, x_dtype=0, w_dtype=0, y_dtype=0, rows=7, cols=cols, eps=EPS, dx=dx))
    fine = [0, 1, 2, 3, 6]
    mira.mira_rmsnorm_grad(mira.RmsNormGradArgs(dy=dy, h=x, weight=w, x_dtype=0, w_dtype=0, y_dtype=0, rows=4, cols=cols, eps=EPS, dweight=dw,
                                                workspace=ws, workspace_bytes=nb))
    torch.cuda.synchronize()
    h = f64(x)
    want, _ = norm(h[fine], 1.0, EPS)
    chain = 8 * -(-cols // 8192) + 40
    assert (np.abs(f64(y)[fine] - want) <= chain * U32 * np.abs(want)).all()
    assert (f64(y)[0] == 0).all() and (q[0] == 0).all()
    assert np.isnan(f64(y)[4]).all()
    assert np.isnan(f64(y)[5, -1]) and (f64(y)[5, :-1] == 0).all()
    gx, gw, terms, wmag = norm_grad(f64(dy)[fine], None, h[fine], np.ones(cols), EPS)
    assert (np.abs(f64(dx)[fine] - gx) <= 3 * chain * U32 * terms + 1e-37).all()
    _, gw, _, wmag = norm_grad(f64(dy)[:4], None, h[:4], np.ones(cols), EPS)
    assert (np.abs(f64(dw) - gw) <= (chain + 30) * U32 * wmag).all()
    assert np.isnan(f64(dx)[4]).all()


@pytest.mark.parametrize("rows,cols", SIZES + [(5000, 300), (3000, 1000), (2500, 2000), (1200, 4100)])
@pytest.mark.parametrize("x,w,y,dsum,pad,shift", [("bf16", "bf16", "bf16", True, 0, 0), ("f32", "f32", "f32", False, 0, 0),
                                                  ("bf16", "f32", "f32", False, 3, 1), ("f32", "bf16", "bf16", True, 5, 3)])
def test_gradient(rows, cols, x, w, y, dsum, pad, shift):
    rng = np.random.default_rng([rows, cols, pad, 1])
    H = Guarded(rows, cols, dt(x), cols + pad, shift).put(_rows(rng, rows, cols))
    D = Guarded(rows, cols, dt(y), cols + 2 * pad, shift).put(torch.from_numpy(rng.normal(0, 1, (rows, cols))).cuda())
    S = Guarded(rows, cols, dt(x), cols + pad, shift).put(torch.from_numpy(rng.normal(0, 1, (rows, cols))).cuda())
    W = Guarded(1, cols, dt(w), None, shift).put(1 + 0.2 * torch.from_numpy(rng.normal(0, 1, (1, cols))).cuda())
    DX, DW = Guarded(rows, cols, dt(x), cols + 3 * pad, shift), Guarded(1, cols, torch.float32, None, shift)
    nb = mira.mira_rmsnorm_grad_workspace_bytes(rows, cols)
    ws = Guarded(1, nb, torch.uint8)
    args = mira.RmsNormGradArgs(dy=D.v, dsum=S.v if dsum else None, h=H.v, weight=W.v, x_dtype=code(x), w_dtype=code(w), y_dtype=code(y), rows=rows,
                                cols=cols, eps=EPS, ld_dy=D.ld, ld_dsum=S.ld, ld_h=H.ld, dx=DX.v, ld_dx=DX.ld, dweight=DW.v, workspace=ws.v,
                                workspace_bytes=nb)
    assert ws.v.data_ptr() % 256 == 0
    mira.mira_rmsnorm_grad(args)
    torch.cuda.synchronize()
    assert all(g.intact() for g in (H, D, S, W, DX, DW, ws))
    want, gw, terms, wmag = norm_grad(f64(D.v), f64(S.v) if dsum else None, f64(H.v), f64(W.v), EPS)
    chain = 8 * -(-cols // 8192) + 40
    off = 3 * chain * U32 * terms     # r, the mean of n g (its own sums and r again), and their products
    assert (np.abs(f64(DX.v) - want) <= off + unit(x) * (np.abs(want) + off) + 1e-38).all()
    # a workgroup's rows one after another, four of them, a 16th of the parts, the 16
    assert (np.abs(f64(DW.v)[0] - gw) <= (chain + 8 + min(rows, -(-rows // 64) + 64) + 24) * U32 * wmag + 1e-38).all()
    first = DX.v.clone(), DW.v.clone()
    args.dx = None
    mira.mira_rmsnorm_grad(args)
    args.dx, args.dweight, args.workspace = DX.v, None, None
    DX.v.zero_()
    mira.mira_rmsnorm_grad(args)
    torch.cuda.synchronize()
    assert torch.equal(DX.v, first[0]) and torch.equal(DW.v, first[1])   # alone, the same bits
    if dsum:                                                            # over dsum
        args.dx, args.ld_dx = S.v, S.ld
        mira.mira_rmsnorm_grad(args)
        torch.cuda.synchronize()
        assert torch.equal(S.v, first[0])


def test_gradient_without_rows():
    dw = torch.full((70,), 5.0, device="cuda")
    nb = mira.mira_rmsnorm_grad_workspace_bytes(0, 70)
    mira.mira_rmsnorm_grad(mira.RmsNormGradArgs(rows=0, cols=70, dweight=dw, workspace=torch.empty(nb, dtype=torch.uint8, device="cuda"),
                                                workspace_bytes=nb))
    torch.cuda.synchronize()
    assert (dw == 0).all()


def test_gradient_against_differences():
    """The gradients from central differences of the 64-bit loss sum(g y) + sum(e h)."""
    rows, cols = 5, 37
    rng = np.random.default_rng(2)
    h, g, e = (rng.normal(0, 1, (rows, cols)).astype(np.float32) for _ in range(3))
    w = rng.normal(1, 0.2, cols).astype(np.float32)
    t = [torch.from_numpy(v).cuda() for v in (g, e, h, w)]
    dx, dw = torch.empty(rows, cols, device="cuda"), torch.empty(cols, device="cuda")
    nb = mira.mira_rmsnorm_grad_workspace_bytes(rows, cols)
    mira.mira_rmsnorm_grad(mira.RmsNormGradArgs(dy=t[0], dsum=t[1], h=t[2], weight=t[3], x_dtype=0, w_dtype=0, y_dtype=0, rows=rows, cols=cols, eps=EPS,
                                                dx=dx, dweight=dw, workspace=torch.empty(nb, dtype=torch.uint8, device="cuda"), workspace_bytes=nb))
    torch.cuda.synchronize()
    h, g, e, w = (v.astype(np.float64) for v in (h, g, e, w))

    def loss(h, w):
        return (g * norm(h, w, EPS)[0]).sum() + (e * h).sum()

    step = 1e-5   # differences are off by step^2 times third derivatives (about 10) and 1e-16 / step
    for r, c in [(0, 0), (1, 5), (2, 36), (4, 20)]:
        d = np.zeros_like(h)
        d[r, c] = step
        assert abs((loss(h + d, w) - loss(h - d, w)) / (2 * step) - float(dx[r, c])) < 1e-5
    for c in (0, 7, 36):
        d = np.zeros_like(w)
        d[c] = step
        assert abs((loss(h, w + d) - loss(h, w - d)) / (2 * step) - float(dw[c])) < 1e-5


def test_far_rows():
    """Rows so far apart that offsets pass 2^32 bytes: the same bits as on dense rows."""
    ld, rows, cols = 1 << 27, 20, 300
    rng = np.random.default_rng(5)
    x = _rows(rng, rows, cols).bfloat16()
    far, out = (torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld) for _ in range(2))
    far[:, :cols] = x
    w = torch.ones(cols, dtype=torch.bfloat16, device="cuda")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mira.mira_rmsnorm(mira.RmsNormArgs(x=x, weight=w, rows=rows, cols=cols, y=y))
    mira.mira_rmsnorm(mira.RmsNormArgs(x=far, weight=w, rows=rows, cols=cols, ldx=ld, y=out, ldy=ld))
    torch.cuda.synchronize()
    assert torch.equal(out[:, :cols], y)
    mira.mira_rmsnorm_grad(mira.RmsNormGradArgs(dy=y, h=x, weight=w, rows=rows, cols=cols, dx=dx))
    mira.mira_rmsnorm_grad(mira.RmsNormGradArgs(dy=out, ld_dy=ld, h=far, ld_h=ld, weight=w, rows=rows, cols=cols, dx=out[:, 512:], ld_dx=ld))
    torch.cuda.synchronize()
    assert torch.equal(out[:, 512:512 + cols], dx)
    del far, out
    torch.cuda.empty_cache()


# rows of 16 and 32 lanes and of a wave, at and beside their ends; rows that one workgroup takes in turn
SHORT = [(r, c) for c in (15, 16, 127, 128, 129, 256, 257, 511) for r in (1, 16, 17, 49, 700)]
CHAIN.update({c: 30 for _, c in SHORT})


@pytest.mark.parametrize("rows,cols", SHORT + [(40000, 128), (3, 3000), (4, 3000), (2, 9000)])
@pytest.mark.parametrize("x,w,y,extra,pad,shift", [("bf16", "bf16", "bf16", True, 0, 0), ("f32", "bf16", "f32", False, 3, 1)])
def test_short_rows(rows, cols, x, w, y, extra, pad, shift):
    if (rows, cols) in SHORT:
        test_forward(rows, cols, x, w, y, extra, pad, shift)
    test_gradient(rows, cols, x, w, y, extra, pad, shift)


@pytest.mark.parametrize("cols", [10, 128, 200, 400])
def test_far_and_near_rows_side_by_side(cols):
    """Rows whose squares pass fp32's range beside others, of NaN and infinities too."""
    rng = np.random.default_rng(cols)
    rows = 70
    x = _rows(rng, rows, cols)
    x[1::3] *= 1e30
    bad = list(range(2, rows, 9))
    x[bad, 0] = torch.tensor([float("nan"), float("inf")], device="cuda").repeat(rows)[:len(bad)]
    w = torch.ones(cols, device="cuda")
    y, dx, dy = torch.empty_like(x), torch.empty_like(x), torch.from_numpy(rng.normal(0, 1, (rows, cols))).float().cuda()
    mira.mira_rmsnorm(mira.RmsNormArgs(x=x, weight=w, x_dtype=0, w_dtype=0, y_dtype=0, rows=rows, cols=cols, eps=EPS, y=y))
    mira.mira_rmsnorm_grad(mira.RmsNormGradArgs(dy=dy, h=x, weight=w, x_dtype=0, w_dtype=0, y_dtype=0, rows=rows, cols=cols, eps=EPS, dx=dx))
    fine = [r for r in range(rows) if r not in bad]
    dw, nb = torch.empty(cols, device="cuda"), mira.mira_rmsnorm_grad_workspace_bytes(len(fine), cols)
    mira.mira_rmsnorm_grad(mira.RmsNormGradArgs(dy=dy[fine], h=x[fine], weight=w, x_dtype=0, w_dtype=0, y_dtype=0, rows=len(fine), cols=cols, eps=EPS,
                                                dweight=dw, workspace=torch.empty(nb, dtype=torch.uint8, device="cuda"), workspace_bytes=nb))
    torch.cuda.synchronize()
    want, _ = norm(f64(x)[fine], 1.0, EPS)
    assert (np.abs(f64(y)[fine] - want) <= 30 * U32 * np.abs(want)).all()
    gx, gw, terms, wmag = norm_grad(f64(dy)[fine], None, f64(x)[fine], np.ones(cols), EPS)
    assert (np.abs(f64(dx)[fine] - gx) <= 3 * 48 * U32 * terms + 1e-37).all()
    assert (np.abs(f64(dw) - gw) <= (48 + 70 + 32) * U32 * wmag).all()
    assert np.isnan(f64(y)[bad, 0]).all() and np.isnan(f64(y)[bad[0]]).all() and (f64(y)[bad[1], 1:] == 0).all()


def test_large_calls_repeat_their_bits():
    rows, cols = 4096, 4096
    g = torch.Generator(device="cuda").manual_seed(8)
    x, res, dy = (torch.randn(rows, cols, generator=g, device="cuda").bfloat16() for _ in range(3))
    w = (1 + 0.1 * torch.randn(cols, generator=g, device="cuda")).bfloat16()
    nb = mira.mira_rmsnorm_grad_workspace_bytes(rows, cols)
    ws, out = torch.empty(nb, dtype=torch.uint8, device="cuda"), []
    for _ in range(3):
        s, y, dx = (torch.empty_like(x) for _ in range(3))
        q, scale, dw = torch.empty(rows, cols, dtype=torch.uint8, device="cuda"), torch.empty(rows, cols // 128, device="cuda"), torch.empty(cols, device="cuda")
        mira.mira_rmsnorm(mira.RmsNormArgs(x=x, residual=res, weight=w, rows=rows, cols=cols, sum=s, y=y, q=q, scale=scale))
        mira.mira_rmsnorm_grad(mira.RmsNormGradArgs(dy=dy, dsum=res, h=s, weight=w, rows=rows, cols=cols, dx=dx, dweight=dw, workspace=ws, workspace_bytes=nb))
        out.append((s, y, q, scale, dx, dw))
    torch.cuda.synchronize()
    for o in out[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, out[0]))
