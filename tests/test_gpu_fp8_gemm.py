"""The FP8 product against the 64-bit product of the same bytes and scales:
sizes from one row and column up, odd ones, both output types, strides, groups
with empty ones, gathered rows, rows of no group, NaN, and gradients through the
transposed copy."""
import numpy as np
import pytest
import torch

import paper_2609_38090_amd as mira
from ops_reference import dequantize, gemm, gemm_bound, source_rows

pytestmark = pytest.mark.gpu


def _codes(gen, rows, cols, ld):
    """Random finite e4m3 bytes [rows][ld]: zeros up to a multiple of 16, NaN codes behind it."""
    q = torch.randint(0, 256, (rows, ld), generator=gen, dtype=torch.uint8)
    q[(q & 127) == 127] = 0x35
    c16 = -(-cols // 16) * 16
    q[:, cols:c16] = 0
    q[:, c16:] = 0x7F
    return q


class Case:
    def __init__(self, M, N, K, out="bf16", G=1, sizes=None, lo=0, tail=0, top_k=0, T=0, shared=0, pads=(0, 0, 0, 0, 0), seed=0):
        gen = torch.Generator().manual_seed(hash((M, N, K, G, seed)) % 2 ** 31)
        self.M, self.N, self.K, self.G, self.top_k = M, N, K, G, top_k
        self.tdt = torch.float32 if out == "f32" else torch.bfloat16
        k16, kb, nb = -(-K // 16) * 16, -(-K // 128), -(-N // 128)
        self.ldx, self.ldw, self.ld_xs, self.ld_ws, self.ldo = k16 + 16 * pads[0], k16 + 16 * pads[1], kb + pads[2], kb + pads[3], N + pads[4]
        self.x_rows = T if top_k else M
        self.x = _codes(gen, max(1, self.x_rows), K, self.ldx)
        self.w = _codes(gen, G * N, K, self.ldw).view(G, N, self.ldw)
        ln = lambda *s: torch.exp(torch.randn(*s, generator=gen))  # noqa: E731
        self.xs, self.ws = ln(max(1, self.x_rows), self.ld_xs) * 0.01, ln(G, nb, self.ld_ws) * 0.001
        self.off, self.order = None, None
        if sizes is not None:
            self.off = torch.tensor(np.concatenate([[lo], lo + np.cumsum(sizes)]), dtype=torch.int32)
            assert int(self.off[-1]) + tail == M
        if top_k:
            pairs = T * top_k + shared * T
            self.order = torch.randint(0, pairs, (M,), generator=gen, dtype=torch.int32)

    def run(self, stream=None):
        d = {n: getattr(self, n).cuda() if getattr(self, n) is not None else None for n in ("x", "w", "xs", "ws", "off", "order")}
        self.out = torch.full((self.M + 1, self.ldo), -77.0, dtype=self.tdt, device="cuda")
        a = mira.Fp8GemmArgs(m=self.M, n=self.N, k=self.K, n_groups=self.G,
                             out_dtype=mira.MIRA_F32 if self.tdt == torch.float32 else mira.MIRA_BF16, x_rows=self.x_rows,
                             top_k=self.top_k, x=d["x"], ldx=self.ldx, x_scale=d["xs"], ld_xs=self.ld_xs, w=d["w"], ldw=self.ldw,
                             w_scale=d["ws"], ld_ws=self.ld_ws, offsets=d["off"], pair_order=d["order"], out=self.out, ldo=self.ldo)
        nb = mira.mira_fp8_gemm_workspace_bytes(a)
        ws = torch.full((nb,), 0xFF, dtype=torch.uint8, device="cuda")
        a.workspace, a.workspace_bytes = ws, nb
        self.keep, self.args = (d, ws), a
        mira.mira_fp8_gemm(a, stream)
        torch.cuda.synchronize()
        return self.out

    def check(self, nan=False):
        out = self.out.double().cpu()
        assert (out[self.M:] == -77).all() and (out[:, self.N:] == -77).all()
        x = dequantize(self.x, self.xs, 1, max(1, self.x_rows), self.K)
        src = torch.arange(self.M) if self.order is None else source_rows(self.order, self.x_rows, self.top_k)
        off = self.off.tolist() if self.off is not None else [0, self.M]
        assert (out[:off[0], :self.N] == -77).all() and (out[off[-1]:self.M, :self.N] == -77).all()
        for g in range(self.G):
            if off[g] == off[g + 1]:
                continue
            r = src[off[g]:off[g + 1]]
            xg = torch.where((r >= 0)[:, None], x[r.clamp(min=0)], torch.zeros(1, dtype=torch.float64))
            w = dequantize(self.w[g], self.ws[g], 128, self.N, self.K)
            want, mag = gemm(xg, w)
            got = out[off[g]:off[g + 1], :self.N]
            assert torch.equal(torch.isnan(got), torch.isnan(want))
            bad = torch.nan_to_num((got - want).abs() - gemm_bound(mag, self.K, self.tdt == torch.bfloat16, want)) > 0
            assert not bad.any(), (g, bad.nonzero()[:5].tolist(), float((got - want).abs().max()))


ROWS = [1, 2, 15, 16, 17, 33, 64, 65, 129, 300]


@pytest.mark.parametrize("M", ROWS)
@pytest.mark.parametrize("N,K", [(1, 1), (16, 128), (130, 200), (100, 1111), (257, 129), (384, 2048)])
def test_sizes(M, N, K):
    c = Case(M, N, K, "f32" if (M + N) % 2 else "bf16")
    c.run()
    c.check()


@pytest.mark.parametrize("M,N,K,out", [(1, 4096, 4096, "bf16"), (1, 64, 14336, "f32"), (8, 5003, 2001, "f32"), (16, 512, 16000, "bf16"),
                                       (40, 1000, 8192, "f32"), (257, 513, 1025, "f32"), (512, 768, 4096, "bf16"), (700, 1300, 640, "f32"),
                                       (1030, 900, 385, "bf16"), (3, 70000, 17, "bf16"), (2100, 2300, 130, "bf16")])
def test_larger(M, N, K, out):
    c = Case(M, N, K, out)
    c.run()
    c.check()


# rows, columns, contraction, groups that the dispatch sends to each tile shape
SHAPES = {"fp8_gemm_256x256": (4100, 8300, 140, 1), "fp8_gemm_256x128": (1900, 4090, 260, 1),
          "fp8_gemm_128x64": (1500, 2000, 500, 1), "fp8_gemm_64x16": (19, 3000, 700, 1), "fp8_gemm_join": (20, 260, 9000, 1),
          "fp8_gemm_few": (11, 3000, 700, 1)}


@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("tail", [0, 77])
def test_every_tile_shape(name, out, tail):
    M, N, K, G = SHAPES[name]
    c = Case(M, N, K + tail, out, pads=(1, 1, 1, 0, 0))
    mira.mira_profile_enable(True)
    mira.mira_profile_read()
    c.run()
    ran = mira.mira_profile_read()
    mira.mira_profile_enable(False)
    assert name in ran, ran
    c.check()


def _ran(c):
    mira.mira_profile_enable(True)
    mira.mira_profile_read()
    c.run()
    ran = mira.mira_profile_read()
    mira.mira_profile_enable(False)
    return set(ran)


# blocks of the contraction: fewer than a workgroup's four waves, a wave's ring not
# full, full, turned over once and more, with an end inside a block
@pytest.mark.parametrize("K", [1, 128, 400, 512, 1030, 2048, 2049, 4000, 4096, 4100, 8100])
@pytest.mark.parametrize("M,sizes,lo,tail,top_k,shared", [(1, None, 0, 0, 0, 0), (2, None, 0, 0, 0, 0), (8, None, 0, 0, 0, 0), (16, None, 0, 0, 0, 0),
                                                          (7, [0, 3, 0, 1, 2], 0, 1, 0, 0), (16, [16], 0, 0, 0, 0),
                                                          (6, [1, 1, 0, 3, 0, 0, 1], 0, 0, 2, 0), (8, [2, 0, 4], 1, 1, 3, 1)])
def test_few_rows(M, sizes, lo, tail, top_k, shared, K):
    c = Case(M, 83, K, "f32" if K % 3 else "bf16", G=len(sizes) if sizes else 1, sizes=sizes, lo=lo, tail=tail, top_k=top_k,
             T=3 if top_k else 0, shared=shared, pads=(1, 1, 1, 2, 3))
    if top_k:
        c.order[M // 2] = -1
    assert ("fp8_gemm_few" in _ran(c)) == (K * max(M, 4) <= 1 << 16)
    c.check()


def test_few_rows_nan():
    # codes of NaN at the start of a row meet only their own column and row
    c = Case(5, 40, 130, "bf16")
    c.w[0, 3, 0], c.w[0, 20, 129], c.x[2, 0] = 0x7F, 0xFF, 0x7F
    assert _ran(c) == {"fp8_gemm_few"}
    c.check()


# either side of each bound of the dispatch
@pytest.mark.parametrize("M,N,K,few", [(16, 4096, 4096, True), (16, 4112, 4096, False), (17, 64, 256, False), (2, 33000, 4200, True),
                                       (3, 33000, 4200, False), (1, 20, 16384, True), (1, 20, 16400, False), (16, 48, 4128, False),
                                       (1, 16 * 1280, 256, True)])
def test_few_rows_bounds(M, N, K, few):
    c = Case(M, N, K, "bf16")
    assert ("fp8_gemm_few" in _ran(c)) == few
    c.check()


@pytest.mark.parametrize("M,N,K", [(1, 200, 300), (20, 65, 1000), (150, 300, 257), (600, 530, 400)])
@pytest.mark.parametrize("pads", [(1, 0, 0, 3, 1), (0, 2, 1, 0, 3), (3, 3, 2, 2, 8)])
def test_strides(M, N, K, pads):
    c = Case(M, N, K, "f32" if pads[0] == 1 else "bf16", pads=pads)
    c.run()
    c.check()


GROUPS = [([1], 0, 0), ([0, 3, 0, 1], 0, 0), ([5, 0, 17, 40], 2, 3), ([0, 0], 0, 4), ([130, 1, 0, 64, 300, 7], 0, 1),
          ([1] * 64, 0, 0), ([2, 0, 1, 3] * 16, 1, 0), ([700, 0, 5], 0, 0), ([16, 32, 48, 256], 0, 0)]


@pytest.mark.parametrize("sizes,lo,tail", GROUPS)
@pytest.mark.parametrize("N,K,out", [(48, 128, "f32"), (200, 700, "bf16"), (300, 1408, "f32")])
def test_groups(sizes, lo, tail, N, K, out):
    c = Case(sum(sizes) + lo + tail, N, K, out, G=len(sizes), sizes=sizes, lo=lo, tail=tail)
    c.run()
    c.check()


# ends on either side of a quarter of a tile, of half and of a whole one; gathered, and rows of no group
@pytest.mark.parametrize("sizes,lo,tail", [([256, 128, 129, 0, 255, 257, 1, 600], 0, 0), ([127, 128, 129, 383, 384, 385], 3, 5), ([63, 64, 65, 0, 319, 320, 321], 0, 0), ([31, 32, 33, 95, 96, 97, 700], 0, 0),
                                           ([1, 2, 3, 1, 1500, 0, 0, 1], 0, 0), ([0, 1500, 0], 0, 130)])
@pytest.mark.parametrize("K,top_k", [(300, 0), (1111, 2), (128, 6)])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_tiles_of_several_heights(sizes, lo, tail, K, top_k, out):
    c = Case(sum(sizes) + lo + tail, 12001, K, out, G=len(sizes), sizes=sizes, lo=lo, tail=tail, top_k=top_k, T=311 if top_k else 0)
    ran = _ran(c)
    assert ran == {"fp8_gemm_mixed"} or (out == "f32" and (K == 128 or len(sizes) == 3))  # (tiles of one height may suit these)
    c.check()


@pytest.mark.parametrize("sizes,lo,tail", GROUPS[1:7])
@pytest.mark.parametrize("T,top_k,shared", [(1, 1, 0), (7, 2, 1), (50, 8, 2)])
def test_gathered_rows(sizes, lo, tail, T, top_k, shared):
    c = Case(sum(sizes) + lo + tail, 150, 384, "f32", G=len(sizes), sizes=sizes, lo=lo, tail=tail, top_k=top_k, T=T, shared=shared)
    c.order[::5] = -1                       # rows of zeros
    c.run()
    c.check()


@pytest.mark.parametrize("M", [3, 20, 200, 600])
def test_one_group_with_offsets_and_gather(M):
    c = Case(M, 140, 500, "f32", G=1, sizes=[M - 2], lo=1, tail=1, top_k=3, T=11)
    c.run()
    c.check()


@pytest.mark.parametrize("M", [1, 7, 40, 300])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_gather_without_offsets_and_rows_of_zeros(M, out):
    c = Case(M, 140, 500, out, top_k=3, T=11)
    c.x[0, 5] = 0x7F  # the row that a row of zeros reads in place of its own
    c.order[::4] = -1
    c.run()
    c.check()
    assert (c.out[:M:4, :140] == 0).all()


@pytest.mark.parametrize("M", [2, 40, 300])
def test_nan_stays_in_its_row_and_column(M):
    c = Case(M, 160, 300, "f32")
    c.x[1, 7] = 0x7F
    c.w[0, 33, 290] = 0xFF
    c.run()
    c.check()
    out = c.out[:M, :160]
    assert torch.isnan(out[1]).all() and torch.isnan(out[:, 33]).all()
    assert int(torch.isnan(out).sum()) == 160 + M - 1


@pytest.mark.parametrize("M", [2, 40, 300])
def test_extreme_scales_and_zero_rows(M):
    c = Case(M, 130, 400, "f32")
    c.x[0] = 0
    c.xs[1] = 1e30
    c.ws[0, 1] = 1e-30
    c.run()
    c.check()
    assert (c.out[0, :130] == 0).all()


@pytest.mark.parametrize("M,N,K", [(1, 256, 4096), (16, 300, 9000), (100, 400, 8192), (700, 512, 512)])
def test_runs_give_the_same_bits(M, N, K):
    c = Case(M, N, K, "f32")
    a = c.run().clone()
    for _ in range(3):
        assert torch.equal(a, c.run())


def test_rows_do_not_depend_on_their_company():
    """A row's result in a call of its own sizes class: the same rows, permuted, give the permuted result."""
    c = Case(200, 300, 700, "f32")
    a = c.run()[:200].clone()
    p = torch.randperm(200, generator=torch.Generator().manual_seed(1))
    c.x, c.xs = c.x[p], c.xs[p]
    assert torch.equal(c.run()[:200], a[p.cuda()])


@pytest.mark.parametrize("M,N,K,G", [(1, 300, 8192, 1), (40, 300, 600, 1), (600, 300, 600, 1), (64, 100, 256, 8), (6, 300, 4100, 3),
                                     (40, 300, 9000, 1), (800, 6000, 700, 4)])
def test_other_stream_and_graph(M, N, K, G):
    c = Case(M, N, K, "f32", G=G, sizes=[M // G] * G if G > 1 else None)
    want = c.run().clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert torch.equal(c.run(stream=side), want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mira.mira_fp8_gemm(c.args)
    for _ in range(4):
        c.out.fill_(-77.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, want)


def test_offsets_that_do_not_ascend_stay_inside_tiles_of_several_heights():
    for off in ([0, 700, 20, 1500, 300], [-5, 10, 99999, 20, 0], [1500, 0, 0, 0, 0], [0, 1500, 0, 1500, 0], [0, 1500, 1500, 0, 1500]):
        for out in ("bf16", "f32"):
            c = Case(1500, 12001, 300, out, G=4, sizes=[375] * 4)
            c.off = torch.tensor(off, dtype=torch.int32)
            assert _ran(c) == {"fp8_gemm_mixed"}
            res = c.out.double().cpu()
            assert (res[c.M:] == -77).all() and (res[:, c.N:] == -77).all()


def test_offsets_that_do_not_ascend_stay_inside_few_rows():
    for off in ([0, 12, 3, 16], [-5, 10, 99999, 20], [16, 0, 0, 0], [0, 16, 0, 16]):
        c = Case(16, 83, 300, "bf16", G=3, sizes=[5, 5, 6])
        c.off = torch.tensor(off, dtype=torch.int32)
        assert _ran(c) == {"fp8_gemm_few"}
        res = c.out.double().cpu()
        assert (res[c.M:] == -77).all() and (res[:, c.N:] == -77).all()


def test_offsets_that_do_not_ascend_stay_inside():
    for off in ([0, 50, 20, 600], [-5, 10, 99999, 20], [600, 0, 0, 0], [0, 600, 0, 600]):
        c = Case(600, 200, 300, "bf16", G=3, sizes=[200, 200, 200])
        c.off = torch.tensor(off, dtype=torch.int32)
        out = c.run()
        assert (out[600:] == -77).all()


@pytest.mark.parametrize("M,N,K", [(3, 96, 160), (70, 300, 200)])
def test_input_gradient_through_the_transposed_copy(M, N, K):
    """dX = dY W as the product of quantized dY with the weight's transposed copy:
    exact against the 64-bit product of the same held values, and against
    differences of the 64-bit forward product."""
    gen = torch.Generator().manual_seed(M)
    w32, dy32 = torch.randn(N, K, generator=gen).cuda(), torch.randn(M, N, generator=gen).cuda()
    pad = lambda n: -(-n // 16) * 16  # noqa: E731
    blk = lambda n: -(-n // 128)  # noqa: E731
    wq, wt = (torch.empty(r, pad(c), dtype=torch.uint8, device="cuda") for r, c in ((N, K), (K, N)))
    s, st = torch.empty(blk(N), blk(K), device="cuda"), torch.empty(blk(K), blk(N), device="cuda")
    mira.mira_fp8_quantize(mira.Fp8QuantArgs(x=w32, x_dtype=mira.MIRA_F32, rows=N, cols=K, block_rows=128, q=wq, scale=s, qt=wt, scale_t=st))
    dq, ds = torch.empty(M, pad(N), dtype=torch.uint8, device="cuda"), torch.empty(M, blk(N), device="cuda")
    mira.mira_fp8_quantize(mira.Fp8QuantArgs(x=dy32, x_dtype=mira.MIRA_F32, rows=M, cols=N, q=dq, scale=ds))
    dx = torch.empty(M, K, device="cuda")
    a = mira.Fp8GemmArgs(m=M, n=K, k=N, out_dtype=mira.MIRA_F32, x_rows=M, x=dq, x_scale=ds, w=wt, w_scale=st, out=dx)
    nb = mira.mira_fp8_gemm_workspace_bytes(a)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = ws, nb
    mira.mira_fp8_gemm(a)
    torch.cuda.synchronize()
    dy, w = dequantize(dq, ds, 1, M, N).cpu(), dequantize(wq, s, 128, N, K).cpu()
    want, mag = dy @ w, dy.abs() @ w.abs()
    assert ((dx.double().cpu() - want).abs() <= gemm_bound(mag, N, False, want)).all()
    # L = sum(dY * (X W^T)) is linear in X: a difference over any step is the gradient
    x = torch.randn(M, K, generator=gen, dtype=torch.float64)
    for i, j in ((0, 0), (M - 1, K - 1), (M // 2, 7)):
        e = torch.zeros_like(x)
        e[i, j] = 0.5
        diff = ((dy * ((x + e) @ w.t())).sum() - (dy * ((x - e) @ w.t())).sum())
        tol = gemm_bound(mag, N, False, want)[i, j] + 4 * N * M * K * 2.0 ** -52 * float((dy.abs() * (x.abs() @ w.abs().t())).max())
        assert abs(float(dx[i, j]) - float(diff)) <= float(tol)


def test_two_streams_at_once():
    """Calls of every tile shape and of parts, each on its own buffers, in flight together."""
    cases = [Case(M, N, K, out) for M, N, K, out in ((2050, 4096, 300, "bf16"), (40, 300, 9000, "f32"), (600, 1000, 700, "f32"), (3, 5000, 900, "bf16"))]
    want = [c.run().clone() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(3):
        for c in cases:
            c.out.fill_(-77.0)
        torch.cuda.synchronize()
        for c, st in zip(cases, streams):
            mira.mira_fp8_gemm(c.args, st)
        torch.cuda.synchronize()
        for c, w in zip(cases, want):
            assert torch.equal(c.out, w)


@pytest.mark.parametrize("M,N,K", [(37, 77, 300), (600, 514, 700)])
@pytest.mark.parametrize("shift", [1, 2, 3, 8])
def test_out_of_any_alignment(M, N, K, shift):
    """out starting `shift` elements past an aligned address, rows of odd length."""
    for out in ("bf16", "f32"):
        c = Case(M, N, K, out, pads=(0, 0, 0, 0, 3))
        c.run()
        want = c.out[:M, :N].clone()
        flat = torch.full((M * (N + 3) + 16,), -5.0, dtype=c.tdt, device="cuda")
        c.args.out = flat[shift:]
        mira.mira_fp8_gemm(c.args)
        torch.cuda.synchronize()
        got = flat[shift:shift + M * (N + 3)].view(M, N + 3)
        assert torch.equal(got[:, :N], want) and (got[:, N:] == -5).all()
        assert (flat[:shift] == -5).all() and (flat[shift + M * (N + 3):] == -5).all()


# groups whose contraction is split into parts that a second launch adds (sizes, rows of no
# group before and behind, columns, contraction): several groups, empty ones, one group of
# nearly all rows, dense rows and gathered ones, shared pairs, rows of zeros
@pytest.mark.parametrize("sizes,lo,tail,N,K", [
    ([5, 0, 3, 7, 0, 0, 1, 9, 2, 0, 4, 3, 0, 1], 3, 4, 417, 9100), ([20, 0, 60, 17], 0, 0, 130, 9000), ([0, 0, 90, 0], 5, 2, 300, 8200),
    ([70, 130, 0, 200, 31, 65, 100, 0, 64, 84], 0, 0, 381, 4693), ([37], 2, 1, 260, 9001)])
@pytest.mark.parametrize("top_k,shared", [(0, 0), (2, 1)])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_groups_in_parts(sizes, lo, tail, N, K, top_k, shared, out):
    c = Case(sum(sizes) + lo + tail, N, K, out, G=len(sizes), sizes=sizes, lo=lo, tail=tail, top_k=top_k, T=29 if top_k else 0,
             shared=shared, pads=(1, 1, 1, 2, 3))
    if top_k:
        c.x[0, 5] = 0x7F  # the row that a row of zeros reads in place of its own
        c.order[::5] = -1
    assert "fp8_gemm_join" in _ran(c)
    c.check()
    if top_k:
        at = torch.arange(lo, c.M - tail)
        assert (c.out[at[at % 5 == 0].cuda(), :N] == 0).all()


def test_groups_in_parts_captured():
    c = Case(42, 449, 6136, "f32", G=4, sizes=[20, 0, 3, 15], lo=1, tail=3, top_k=3, T=17, shared=1)
    c.order[::5] = -1
    assert "fp8_gemm_join" in _ran(c)
    c.check()
    want = c.out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mira.mira_fp8_gemm(c.args)
    for _ in range(4):
        c.out.fill_(-77.0)
        c.keep[1].fill_(0xFF)  # the workspace's content does not matter
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, want)


def test_parts_write_only_their_workspace():
    """The workspace in the middle of a buffer, and offsets that do not ascend."""
    for off in (None, [0, 12, 3, 40], [-5, 10, 99999, 20], [40, 0, 0, 0], [0, 40, 0, 40]):
        c = Case(40, 260, 9000, "f32", G=3 if off else 1, sizes=[13, 13, 14] if off else None)
        if off:
            c.off = torch.tensor(off, dtype=torch.int32)
        assert "fp8_gemm_join" in _ran(c)
        nb = c.args.workspace_bytes
        assert nb > 0
        guard = torch.full((nb + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
        c.args.workspace = guard[4096:]
        assert c.args.workspace.data_ptr() % 256 == 0
        mira.mira_fp8_gemm(c.args)
        torch.cuda.synchronize()
        assert (guard[:4096] == 0xA5).all() and (guard[4096 + nb:] == 0xA5).all()
        out = c.out
        assert (out[c.M:] == -77).all() and (out[:, c.N:] == -77).all()
        if not off:
            c.check()


@pytest.mark.parametrize("N,K,sizes", [(96, 160, [3, 0, 1, 12]), (300, 200, [70, 1, 0, 200]), (260, 9000, [5, 0, 9])])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_input_gradient_of_groups_through_the_transposed_copies(N, K, sizes, out):
    """dX = dY W_g of each group's rows: the grouped product on the experts' transposed
    copies, against the 64-bit product of the values that the plain copies hold."""
    G, M = len(sizes), sum(sizes)
    gen = torch.Generator().manual_seed(N)
    pad = lambda n: -(-n // 16) * 16  # noqa: E731
    blk = lambda n: -(-n // 128)  # noqa: E731
    u8 = lambda *s: torch.empty(*s, dtype=torch.uint8, device="cuda")  # noqa: E731
    wq, wt, s, st = u8(G, N, pad(K)), u8(G, K, pad(N)), torch.empty(G, blk(N), blk(K), device="cuda"), torch.empty(G, blk(K), blk(N), device="cuda")
    for g in range(G):
        mira.mira_fp8_quantize(mira.Fp8QuantArgs(x=torch.randn(N, K, generator=gen).cuda(), x_dtype=mira.MIRA_F32, rows=N, cols=K, block_rows=128,
                                                 q=wq[g], scale=s[g], qt=wt[g], scale_t=st[g]))
    dq, ds = u8(M, pad(N)), torch.empty(M, blk(N), device="cuda")
    mira.mira_fp8_quantize(mira.Fp8QuantArgs(x=torch.randn(M, N, generator=gen).bfloat16().cuda(), rows=M, cols=N, q=dq, scale=ds))
    off = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32)
    tdt, dt = (torch.float32, mira.MIRA_F32) if out == "f32" else (torch.bfloat16, mira.MIRA_BF16)
    off_dev, dx = off.cuda(), torch.empty(M, K, dtype=tdt, device="cuda")
    a = mira.Fp8GemmArgs(m=M, n=K, k=N, n_groups=G, out_dtype=dt, x_rows=M, x=dq, x_scale=ds, w=wt, w_scale=st, offsets=off_dev, out=dx)
    nb = mira.mira_fp8_gemm_workspace_bytes(a)
    ws = u8(nb)
    a.workspace, a.workspace_bytes = ws, nb
    mira.mira_fp8_gemm(a)
    torch.cuda.synchronize()
    dy = dequantize(dq, ds, 1, M, N).cpu()
    for g in range(G):
        w, at = dequantize(wq[g], s[g], 128, N, K).cpu(), slice(int(off[g]), int(off[g + 1]))
        want, mag = dy[at] @ w, dy[at].abs() @ w.abs()
        assert ((dx[at].double().cpu() - want).abs() <= gemm_bound(mag, N, out == "bf16", want)).all()
