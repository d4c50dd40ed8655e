"""SwiGLU's gradient against 64 bits: types, odd sizes, strides, e4m3 blocks that
straddle gate and up, gates at the ends of the range."""
import numpy as np
import pytest
import torch

import paper_2609_38090_amd as mira
from layer_reference import U32, Guarded, code, dt, e4m3_close, f64, swiglu_grad, unit
from ops_reference import TABLE

pytestmark = pytest.mark.gpu
SIZES = [(1, 1), (1, 128), (3, 127), (5, 129), (2, 64), (17, 1000), (301, 1001), (7, 1408), (4, 14336), (2, 20001), (600, 40), (3, 9001), (5, 520), (9, 65),
         (3, 8193), (2, 16383), (6, 512), (6, 511), (5, 7)]
# exp 4 half steps (and of its rounded sum), the reciprocal 2, 1 - s 2 more, three products; beside the terms' magnitude
STEPS = 16


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("x,d,outs,pad,shift", [("bf16", "bf16", "q", 0, 0), ("f32", "f32", "dx", 0, 0), ("bf16", "f32", "dxq", 3, 1),
                                                ("f32", "bf16", "dxq", 5, 3)])
def test_gradient(rows, cols, x, d, outs, pad, shift):
    rng = np.random.default_rng([rows, cols, pad])
    X = Guarded(rows, 2 * cols, dt(x), 2 * cols + pad, shift).put(torch.from_numpy(rng.normal(0, 4, (rows, 2 * cols))).cuda())
    D = Guarded(rows, cols, dt(d), cols + pad, shift).put(torch.from_numpy(rng.normal(0, 0.1, (rows, cols))).cuda())
    c16, nb = -(-2 * cols // 16) * 16, -(-2 * cols // 128)
    DX = Guarded(rows, 2 * cols, dt(x), 2 * cols + 2 * pad, shift)
    Q, C = Guarded(rows, c16, torch.uint8, c16 + 16 * (pad % 2)), Guarded(rows, nb, torch.float32, nb + pad)
    has_dx, has_q = "dx" in outs, "q" in outs
    mira.mira_swiglu_grad(mira.SwigluGradArgs(x=X.v, dact=D.v, x_dtype=code(x), d_dtype=code(d), rows=rows, cols=cols, q_eps=1e-8, ldx=X.ld,
                                              ld_dact=D.ld, dx=DX.v if has_dx else None, ld_dx=DX.ld, q=Q.v if has_q else None, ldq=Q.ld,
                                              scale=C.v if has_q else None, ld_scale=C.ld))
    torch.cuda.synchronize()
    assert all(g.intact() for g in (X, D, DX, Q, C))
    xs, dd = f64(X.v), f64(D.v)
    dg, du, mag = swiglu_grad(xs[:, :cols], xs[:, cols:], dd)
    want, off = np.concatenate([dg, du], 1), STEPS * U32 * np.concatenate([mag, np.abs(du)], 1)
    if has_dx:
        assert (np.abs(f64(DX.v) - want) <= off + unit(x) * (np.abs(want) + off) + 1e-38).all()
    if has_q:
        q, scale = Q.v.cpu().numpy(), C.v.cpu().numpy()
        assert (q[:, 2 * cols:] == 0).all()
        full = np.zeros((rows, nb * 128))
        full[:, :2 * cols] = np.abs(want)
        a = np.maximum(full.reshape(rows, nb, 128).max(2), 1e-8) / 448
        worst = np.zeros((rows, nb * 128))
        worst[:, :2 * cols] = off
        assert (np.abs(scale - a) <= 2 * U32 * a + worst.reshape(rows, nb, 128).max(2) / 448).all()
        assert e4m3_close(q[:, :2 * cols], scale, want, TABLE, off).all()


@pytest.mark.parametrize("q", [False, True])
def test_gates_at_the_ends(q):
    """Gates over the whole range: where exp(-gate) overflows fp32, where 1 - s is nothing, zero, infinite."""
    gate = torch.cat([torch.linspace(-110, 110, 2201), torch.tensor([-1e30, -3.4e38, 1e30, 3.4e38, 0.0, -0.0, 1e-40, float("inf"), float("-inf"),
                                                                  float("nan")])]).cuda()
    cols = gate.numel()
    x = torch.cat([gate, torch.full((cols,), 1.5, device="cuda")])[None].contiguous()
    d = torch.full((1, cols), -2.0, device="cuda")
    dx = torch.empty_like(x)
    nb = -(-2 * cols // 128)
    mira.mira_swiglu_grad(mira.SwigluGradArgs(x=x, dact=d, x_dtype=0, d_dtype=0, rows=1, cols=cols, dx=dx,
                                              q=torch.empty(1, -(-2 * cols // 16) * 16, dtype=torch.uint8, device="cuda") if q else None,
                                              scale=torch.empty(1, nb, device="cuda") if q else None))
    torch.cuda.synchronize()
    g, u = f64(dx)[0, :cols], f64(dx)[0, cols:]
    with np.errstate(all="ignore"):
        wg, wu, mag = swiglu_grad(f64(gate), 1.5, -2.0)
    n = cols - 3
    # (below 2^-126 s is nothing; its gate times d is at most 2^8 of that)
    assert (np.abs(g[:n] - wg[:n]) <= STEPS * U32 * mag[:n] + 2.0 ** -116).all()
    assert (np.abs(u[:n] - wu[:n])[np.abs(wu[:n]) < 3e38] <= (STEPS * U32 * np.abs(wu[:n]) + 2.0 ** -116)[np.abs(wu[:n]) < 3e38]).all()
    assert np.isnan(g[n:]).all() and np.isinf(u[n]) and np.isnan(u[n + 1:]).all()


def test_far_rows():
    ld, rows, cols = 1 << 27, 20, 130
    rng = np.random.default_rng(7)
    x, d = (torch.from_numpy(rng.normal(0, 2, (rows, n))).cuda().bfloat16() for n in (2 * cols, cols))
    far = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld)
    far[:, :2 * cols], far[:, 512:512 + cols] = x, d
    out = [[torch.empty_like(x), torch.empty(rows, 272, dtype=torch.uint8, device="cuda"), torch.empty(rows, 3, device="cuda")] for _ in range(2)]
    mira.mira_swiglu_grad(mira.SwigluGradArgs(x=x, dact=d, rows=rows, cols=cols, dx=out[0][0], q=out[0][1], scale=out[0][2]))
    mira.mira_swiglu_grad(mira.SwigluGradArgs(x=far, ldx=ld, dact=far[:, 512:], ld_dact=ld, rows=rows, cols=cols, dx=far[:, 1024:], ld_dx=ld, q=out[1][1],
                                              scale=out[1][2]))
    torch.cuda.synchronize()
    assert torch.equal(far[:, 1024:1024 + 2 * cols], out[0][0]) and torch.equal(out[0][1], out[1][1]) and torch.equal(out[0][2], out[1][2])
    del far
    torch.cuda.empty_cache()


@pytest.mark.parametrize("cols", [1, 8, 63, 64, 65, 100, 127, 129, 136, 190, 192, 255, 257, 500])
@pytest.mark.parametrize("rows", [1, 15, 17, 333])
def test_short_rows(rows, cols):
    """Rows of 16 and 32 lanes and of a wave, several to a workgroup."""
    test_gradient(rows, cols, "bf16", "f32", "dxq", 3, 1)
    test_gradient(rows, cols, "f32", "bf16", "q", 0, 0)


@pytest.mark.parametrize("cols", [40, 200, 256, 300, 1001, 16500])
@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_products_beyond_the_range(cols, name):
    """dact up alone passes fp32's range, or falls below it, where dgate does not; dx, and blocks of e4m3."""
    gates = [-100.0, -89.5, -88.0, -80.0, -60.0, -30.0, -3.0, 0.0, 2.5, 50.0]
    factors = [(1e20, 3e19), (3e38, 2.0), (2.0, -3e38), (1e38, 1e10), (-1e10, 1e38), (1e-25, 3e25), (1e-8, 1e30), (1e30, -1e-8), (1e-30, 1e-20),
               (2e38, 0.5), (3.3e38, 0.75), (0.0, 3e38), (1e35, 1e25), (2e38, 2e38)]
    all_of = np.array([(g, d, u) for g in gates for d, u in factors])
    wg, wu, _ = swiglu_grad(all_of[:, 0], all_of[:, 2], all_of[:, 1])
    all_of = all_of[(np.abs(wg) < 3e38) & (np.abs(wu) < 3e38)]
    at = all_of[np.arange(2 * cols).reshape(2, cols) % len(all_of)]
    assert (np.abs(at[:, :, 1] * at[:, :, 2]) > 3.5e38).any()
    x = torch.from_numpy(np.concatenate([at[:, :, 0], at[:, :, 2]], 1)).to(dt(name)).cuda()
    d = torch.from_numpy(at[:, :, 1]).to(dt(name)).cuda()
    wg, wu, mag = swiglu_grad(f64(x)[:, :cols], f64(x)[:, cols:], f64(d))
    want = np.concatenate([wg, wu], 1)
    # s below 2^-126 is nothing: its factors are off by that much
    lost = 2.0 ** -126 * (f64(x)[:, :cols] < -87)
    gate, up, dd = f64(x)[:, :cols], f64(x)[:, cols:], f64(d)
    off = np.concatenate([STEPS * U32 * mag + lost * (1 + np.abs(gate)) * np.abs(up * dd), STEPS * U32 * np.abs(wu) + lost * np.abs(gate * dd)], 1) + 2.0 ** -147
    nb = -(-2 * cols // 128)
    dx, dx2, q = torch.empty_like(x), torch.empty_like(x), torch.empty(2, -(-2 * cols // 16) * 16, dtype=torch.uint8, device="cuda")
    scale = torch.empty(2, nb, device="cuda")
    base = dict(x=x, dact=d, x_dtype=code(name), d_dtype=code(name), rows=2, cols=cols)
    mira.mira_swiglu_grad(mira.SwigluGradArgs(dx=dx, **base))
    mira.mira_swiglu_grad(mira.SwigluGradArgs(dx=dx2, q=q, scale=scale, **base))
    torch.cuda.synchronize()
    assert torch.equal(dx, dx2)
    # bf16 below 2^-126 has steps of 2^-133, of which a rounding is half: 1.4e-41 of these values, for one, is 0 in bf16
    least = 0.0 if name == "f32" else 2.0 ** -134
    assert (np.abs(f64(dx) - want) <= off + least + unit(name) * (np.abs(want) + off)).all()
    full = np.zeros((2, nb * 128))
    full[:, :2 * cols] = np.abs(want)
    a = np.maximum(full.reshape(2, nb, 128).max(2), 1e-8) / 448
    full[:, :2 * cols] = off
    s = f64(scale)
    assert (np.abs(s - a) <= 2 * U32 * a + full.reshape(2, nb, 128).max(2) / 448).all()
    assert e4m3_close(q.cpu().numpy()[:, :2 * cols], scale.cpu().numpy(), want, TABLE, off).all()


def test_large_calls_repeat_their_bits():
    g = torch.Generator(device="cuda").manual_seed(8)
    for rows, cols in ((8192, 14336), (3000, 13399)):
        x, d = (torch.randn(rows, n, generator=g, device="cuda").bfloat16() for n in (2 * cols, cols))
        out = [(torch.empty(rows, -(-2 * cols // 16) * 16, dtype=torch.uint8, device="cuda"), torch.empty(rows, -(-2 * cols // 128), device="cuda"))
               for _ in range(3)]
        for q, scale in out:
            mira.mira_swiglu_grad(mira.SwigluGradArgs(x=x, dact=d, rows=rows, cols=cols, q=q, scale=scale))
        torch.cuda.synchronize()
        for q, scale in out[1:]:
            assert torch.equal(q, out[0][0]) and torch.equal(scale, out[0][1])
