"""The FP8 quantizer byte for byte against the definition (rows and blocks, both
input types, odd sizes, strides), its transposed copy, and SwiGLU within half a
step of e4m3."""
import numpy as np
import pytest
import torch

import paper_2609_38090_amd as mira
from ops_reference import TABLE, U32, quantize

pytestmark = pytest.mark.gpu
EPS = 1e-8


def _input(rng, rows, cols, dt, pad, tweak=None):
    x = rng.normal(0, 1, (rows, cols)).astype(np.float32) * np.exp(rng.normal(0, 2, (rows, 1))).astype(np.float32)
    if tweak:
        tweak(x)
    t = torch.full((rows, cols + pad), 3e4, dtype=torch.float32 if dt == "f32" else torch.bfloat16)
    t[:, :cols] = torch.from_numpy(x)
    return t.cuda(), t[:, :cols].float().numpy()


def _run(x, rows, cols, dt, block, ldx=0, flags=0, qpad=0, spad=0, both=False, stream=None):
    c16, r16, nr, nc = -(-cols // 16) * 16, -(-rows // 16) * 16, -(-rows // block), -(-cols // 128)
    q = torch.full((rows + 1, c16 + qpad), 0xEE, dtype=torch.uint8, device="cuda")
    s = torch.full((nr + 1, nc + spad), -3.0, device="cuda")
    qt = torch.full((cols + 1, r16 + qpad), 0xEE, dtype=torch.uint8, device="cuda") if both else None
    st = torch.full((nc + 1, nr + spad), -3.0, device="cuda") if both else None
    a = mira.Fp8QuantArgs(x=x, x_dtype=mira.MIRA_F32 if dt == "f32" else mira.MIRA_BF16, rows=rows, cols=cols,
                          block_rows=block, eps=EPS, flags=flags, ldx=ldx, q=q, ldq=c16 + qpad, scale=s,
                          ld_scale=nc + spad, qt=qt, ldqt=(r16 + qpad) if both else 0, scale_t=st,
                          ld_scale_t=(nr + spad) if both else 0)
    mira.mira_fp8_quantize(a, stream)
    torch.cuda.synchronize()
    for t, n, live, pad in ((q, rows, cols, c16), (qt, cols, rows, r16)):
        if t is not None:
            assert (t[n:] == 0xEE).all() and (t[:, pad:] == 0xEE).all()   # nothing beyond
            assert (t[:n, live:pad] == 0).all()                           # padding to 16 is zero
    assert (s[nr:] == -3).all() and (s[:, nc:] == -3).all()
    return q, s[:nr, :nc], qt, st, a


SIZES = [(1, 1), (1, 4096), (3, 127), (5, 128), (2, 129), (17, 1000), (130, 384), (8, 4100), (301, 2001), (64, 14336), (1, 16), (33, 40)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dt,pad,qpad,spad", [("f32", 0, 0, 0), ("bf16", 0, 16, 3), ("f32", 5, 16, 0), ("bf16", 3, 0, 1), ("bf16", 8, 32, 0)])
@pytest.mark.parametrize("block", [1, 128])
def test_bytes(rows, cols, dt, pad, qpad, spad, block):
    rng = np.random.default_rng([rows, cols, pad])
    x, x32 = _input(rng, rows, cols, dt, pad)
    both = block == 128 and qpad != 32
    q, s, qt, st, _ = _run(x, rows, cols, dt, block, cols + pad, qpad=qpad, spad=spad, both=both)
    want, scale = quantize(x32, block, EPS)
    assert np.array_equal(s.cpu().numpy(), scale)
    assert np.array_equal(q[:rows, :cols].cpu().numpy(), want)
    if both:
        assert np.array_equal(qt[:cols, :rows].cpu().numpy(), want.T)
        assert np.array_equal(st[:scale.shape[1], :scale.shape[0]].cpu().numpy(), scale.T)


@pytest.mark.parametrize("block", [1, 128])
def test_unaligned_start(block):
    """x one element past an aligned address, rows of odd length."""
    rng = np.random.default_rng(3)
    rows, cols = 20, 301
    flat = torch.from_numpy(rng.normal(0, 1, rows * cols + 1).astype(np.float32)).cuda()
    for dt in ("f32", "bf16"):
        f = flat if dt == "f32" else flat.bfloat16()
        q, s, *_ = _run(f[1:], rows, cols, dt, block)
        want, scale = quantize(f[1:].float().cpu().numpy().reshape(rows, cols), block, EPS)
        assert np.array_equal(q[:rows, :cols].cpu().numpy(), want) and np.array_equal(s.cpu().numpy(), scale)


@pytest.mark.parametrize("block", [1, 128])
def test_special_values(block):
    def tweak(x):
        x[0, :] = 0.0                       # a block of zeros: eps decides its scale
        x[1, :] = 1e-30                     # below eps
        x[2, :128] = 3.0e38                 # near the type's largest
        x[3, 5] = np.nan                    # stays at its place
        x[4, 130] = np.inf                  # its block is lost, the others are not
        x[5, :128] = np.linspace(0, 448, 128)
    rng = np.random.default_rng(5)
    x, x32 = _input(rng, 300 if block == 128 else 6, 300, "f32", 0, tweak)
    rows = x32.shape[0]
    q, s, *_ = _run(x, rows, 300, "f32", block)
    want, scale = quantize(x32, block, EPS)
    v, w = TABLE[q[:rows, :300].cpu().numpy()], TABLE[want]
    with np.errstate(invalid="ignore"):
        r = np.arange(rows) // block
        c = np.arange(300) // 128
        v, w = v * s.cpu().numpy().astype(np.float64)[r][:, c], w * scale.astype(np.float64)[r][:, c]
    assert np.array_equal(np.isnan(v), np.isnan(w))
    assert np.array_equal(np.nan_to_num(v), np.nan_to_num(w))
    assert np.isnan(v[3, 5]) and np.isnan(v[4, 128:256]).all()
    assert np.isfinite(v[4, 256:]).all()
    if block == 1:
        assert (v[0] == 0).all() and np.isnan(v[3]).sum() == 1


@pytest.mark.parametrize("rows,cols,dt,pad", [(1, 64, "f32", 0), (5, 200, "bf16", 0), (33, 1408, "bf16", 8), (7, 301, "f32", 1),
                                              (130, 999, "bf16", 3), (2, 14336, "f32", 0)])
def test_swiglu(rows, cols, dt, pad):
    rng = np.random.default_rng([rows, cols])
    x, x32 = _input(rng, rows, 2 * cols, dt, pad, lambda x: x.__imul__(2.0))
    q, s, *_ = _run(x, rows, cols, dt, 1, 2 * cols + pad, mira.MIRA_FP8_SWIGLU)
    g, u = x32[:, :cols].astype(np.float64), x32[:, cols:].astype(np.float64)
    with np.errstate(over="ignore"):
        h = g / (1 + np.exp(-g)) * u
    nc = -(-cols // 128)
    full = np.zeros((rows, nc * 128))
    full[:, :cols] = h
    scale = np.maximum(np.abs(full).reshape(rows, nc, 128).max(2), EPS) / 448
    # h: exp within 2 steps, a sum, a quotient, a product: 8 half steps; the scale one more
    assert (np.abs(s.cpu().numpy() - scale) <= 10 * U32 * scale).all()
    sc = s.cpu().numpy().astype(np.float64).repeat(128, 1)[:, :cols]
    got = TABLE[q[:rows, :cols].cpu().numpy()] * sc
    # e4m3: half a step is 2^-4 of the value, 2^-10 of the scale among the smallest;
    # h, the inverse and the product before it: 8 + 3 half steps of fp32
    tol = (2.0 ** -4 * np.abs(h) * (1 + 2.0 ** -10) + 2.0 ** -10 * sc) + 12 * U32 * np.abs(h)
    assert (np.abs(got - h) <= tol).all()


def test_swiglu_of_large_gates():
    """exp(-g) beyond the type's range gives 0, not NaN."""
    x = torch.zeros(2, 256, device="cuda")
    x[0, :128], x[0, 128:] = -1000.0, 3.0
    x[1, :128], x[1, 128:] = 1000.0, 3.0
    q, s, *_ = _run(x, 2, 128, "f32", 1, 256, mira.MIRA_FP8_SWIGLU)
    v = TABLE[q[:2, :128].cpu().numpy()] * s.cpu().numpy().astype(np.float64)
    assert (v[0] == 0).all() and np.allclose(v[1], 3000.0, rtol=2 * U32, atol=0)


def test_other_stream_and_graph():
    rng = np.random.default_rng(9)
    x, x32 = _input(rng, 140, 500, "bf16", 0)
    for block in (1, 128):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        q, s, qt, st, a = _run(x, 140, 500, "bf16", block, both=block == 128, stream=side)
        want = [t.clone() for t in (q, s) + ((qt, st) if block == 128 else ())]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            mira.mira_fp8_quantize(a)
        for _ in range(4):
            q[:140, :512].zero_()
            s.zero_()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(u, v) for u, v in zip(want, (q, s, qt, st)))


def _swiglu_rows(gates, ups, dt):
    """One block a row: gate and up at column 5, gates of 0.5 and ups of 1 beside them;
    the quantized values, the scales and the inputs as held, in 64 bits."""
    n = len(gates)
    x = torch.full((n, 256), 0.5)
    x[:, 128:] = 1.0
    x[:, 5], x[:, 133] = torch.tensor(gates, dtype=torch.float32), torch.tensor(ups, dtype=torch.float32)
    x = x.to(torch.float32 if dt == "f32" else torch.bfloat16).cuda()
    q, s, *_ = _run(x, n, 128, dt, 1, 256, mira.MIRA_FP8_SWIGLU)
    s = s.cpu().numpy().astype(np.float64)
    held = x.double().cpu().numpy()
    return TABLE[q[:n, :128].cpu().numpy()], s[:, 0], held[:, 5], held[:, 133]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_swiglu_of_gates_up_to_the_largest(dt):
    """g / (1 + exp(-g)) is g where exp(-g) is nothing beside 1, up to the largest gates;
    an infinity, or a product beyond the range, loses its block; 0 times it only its place."""
    top = 3.38e38  # below the largest value of both types
    gates = [88.0, 200.0, 1e30, 2.3e38, 2.4e38, 2.5e38, 3e38, top, -88.0, -1e30, -2.5e38, -top]
    ups = [0.5, -2.0, 1e-30, 0.5, 1e-3, 0.5, -0.25, 1.0, 1.0, 1.0, 1e3, -0.5]
    v, s, g, u = _swiglu_rows(gates, ups, dt)
    rest = 0.5 / (1 + np.exp(-0.5))
    with np.errstate(over="ignore"):
        want = g / (1 + np.exp(-g)) * u
    scale = np.maximum(np.abs(want), rest) / 448
    # exp within 2 steps, a sum, a quotient, a product, the scale's division: 10 half steps
    assert (np.abs(s - scale) <= 10 * U32 * scale).all()
    got = v[:, 5] * s
    assert (np.abs(got - want) <= (2.0 ** -4 * (1 + 2.0 ** -10) + 12 * U32) * np.abs(want) + 2.0 ** -10 * s).all()
    inf, nan = float("inf"), float("nan")
    v, s, g, u = _swiglu_rows([inf, inf, top, 2.0, 2.0, inf, -inf, nan, 1.0], [0.5, -1e-30, 4.0, inf, -inf, 0.0, 1.0, 1.0, nan], dt)
    assert np.isinf(s[:5]).all() and np.isnan(v[:5, 5]).all()
    assert (np.abs(s[5:] - rest / 448) <= 10 * U32 * rest / 448).all()
    assert np.isnan(v[5:, 5]).all() and np.isfinite(np.delete(v[5:], 5, 1)).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_swiglu_of_gates_whose_exponential_is_near_the_largest(dt):
    """Down to exp(-g) = 2^128 the quotient is held: it is a normal number though
    1 / (1 + exp(-g)) alone is not."""
    gates = [-80.0, -87.0, -87.3, -87.34, -87.5, -88.0, -88.5, -88.7]
    for up in (1e30, -1e35, 3e38):
        v, s, g, u = _swiglu_rows(gates, [up] * len(gates), dt)
        keep = g > -88.72  # (bf16 holds the last one as -88.5)
        assert keep.all()
        want = g / (1 + np.exp(-g)) * u
        scale = np.maximum(np.abs(want), 0.5 / (1 + np.exp(-0.5))) / 448
        # 10 half steps as above, and the reciprocal's, held to 2^-149 of 2^-128: 2^-21
        tol = 10 * U32 + 2.0 ** -21
        assert (np.abs(s - scale) <= tol * scale).all()
        assert (np.abs(v[:, 5] * s - want) <= (2.0 ** -4 * (1 + 2.0 ** -10) + 2 * tol) * np.abs(want) + 2.0 ** -10 * s).all()
