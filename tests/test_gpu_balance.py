"""Balance loss, counts and gradient against the 64-bit statement, by group,
mask, type, stride and odd size; the gradient against differences of the loss."""
import numpy as np
import pytest
import torch

import paper_2609_38090_amd as mira
from ops_reference import U16, U32, balance

pytestmark = pytest.mark.gpu


def _offsets(rng, T, G, edge=0):
    cut = np.sort(rng.integers(edge, T - edge + 1, G - 1)) if G > 1 else np.zeros(0, np.int64)
    return np.concatenate([[edge], cut, [T - edge]]).astype(np.int32)


class Case:
    def __init__(self, T, E, k, G=1, dt="f32", masked=False, pad=0, edge=0, seed=0, tweak=None):
        rng = np.random.default_rng([seed, T, E, k, G])
        self.T, self.E, self.k, self.G = T, E, k, G
        self.tdt = torch.float32 if dt == "f32" else torch.bfloat16
        x = rng.normal(0, 1.5, (T, E)).astype(np.float32)
        self.idx = np.stack([rng.permutation(E)[:k] if E >= k else rng.integers(0, E, k) for _ in range(T)]).astype(np.int32) \
            if T else np.zeros((0, k), np.int32)
        self.mask = (rng.random(T) < 0.7).astype(np.uint8) if masked else None
        self.off = _offsets(rng, T, G, edge) if G > 1 or edge else None
        if tweak:
            tweak(self, x, rng)
        self.coef, self.gl = 0.75, rng.random(G).astype(np.float32) + 0.5
        ld = E + pad
        full = torch.full((max(T, 1), ld), 7.0, dtype=self.tdt)
        full[:T, :E] = torch.from_numpy(x)
        self.logits, self.ld = full.cuda(), ld
        self.x64 = full[:T, :E].double().numpy()

    def run(self, stream=None, **kw):
        c = lambda a, t: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(t).cuda()  # noqa: E731
        self.dev = dict(idx=c(self.idx, torch.int32), off=c(self.off, torch.int32), mask=c(self.mask, torch.uint8),
                        gl=c(self.gl, torch.float32))
        self.out = dict(loss=torch.full((self.G,), 9.0, device="cuda"),
                        counts=torch.full((self.G, self.E), 9, dtype=torch.int32, device="cuda"),
                        mean_prob=torch.full((self.G, self.E), 9.0, device="cuda"),
                        dlogits=torch.full((max(self.T, 1), self.ld), 5.0, dtype=self.tdt, device="cuda"))
        self.out.update(kw)
        nb = mira.mira_balance_workspace_bytes(self.T, self.E, self.G)
        self.ws = torch.full((nb,), 0xAB, dtype=torch.uint8, device="cuda")
        self.args = mira.BalanceArgs(
            logits=self.logits, topk_idx=self.dev["idx"], offsets=self.dev["off"], mask=self.dev["mask"],
            grad_loss=self.dev["gl"], logits_dtype=mira.MIRA_F32 if self.tdt == torch.float32 else mira.MIRA_BF16,
            n_tokens=self.T, n_experts=self.E, top_k=self.k, n_groups=self.G, coef=self.coef, ld_logits=self.ld,
            ld_dlogits=self.ld, workspace=self.ws, workspace_bytes=nb, **self.out)
        mira.mira_balance_loss(self.args, stream)
        torch.cuda.synchronize()
        return self.out

    def check(self):
        out = self.out
        off = self.off if self.off is not None else np.array([0, self.T])
        mask = self.mask if self.mask is not None else np.ones(self.T, np.uint8)
        loss, counts, mean, d = balance(self.x64, self.idx, off, mask, self.coef, self.gl)
        if out["counts"] is not None:
            assert np.array_equal(out["counts"].cpu().numpy(), counts)
        # exp: 2 steps and the rounding of its argument; the row sum's chain of
        # 4 + log2 lanes; reciprocal and product; sums over rows: a lane's chain
        # of at most 600 rows of these sizes, then 16 + 256 partial sums
        finite = self.x64[np.isfinite(self.x64)]
        span = float(finite.max() - finite.min()) if finite.size else 0.0
        ep = (span + 24) * 2 * U32
        es = ep + (600 + 272) * U32
        if out["mean_prob"] is not None:
            got = out["mean_prob"].cpu().numpy().astype(np.float64)
            assert np.array_equal(np.isnan(got), np.isnan(mean))
            np.testing.assert_array_less(np.nan_to_num(np.abs(got - mean)), np.nan_to_num(es * mean) + 1e-37)
        if out["loss"] is not None:
            got = out["loss"].cpu().numpy().astype(np.float64)
            assert np.array_equal(np.isnan(got), np.isnan(loss))
            np.testing.assert_array_less(np.nan_to_num(np.abs(got - loss)), np.nan_to_num((es + 300 * U32) * np.abs(loss)) + 1e-37)
        if out["dlogits"] is not None:
            got = out["dlogits"].double().cpu().numpy()
            assert (got[:, self.E:] == 5.0).all()                 # stride padding untouched
            inside = np.zeros(len(got), bool)
            for g in range(self.G):
                inside[off[g]:off[g + 1]] = True
            assert (got[~inside, :self.E] == 5.0).all()           # rows of no group untouched
            got, want = got[:self.T][inside[:self.T], :self.E], d[inside[:self.T]]
            assert np.array_equal(np.isnan(got), np.isnan(want))
            p = np.exp(self.x64 - np.max(np.where(np.isneginf(self.x64), -1e30, self.x64), 1, keepdims=True)) if self.T else self.x64
            p = (p / np.maximum(p.sum(1, keepdims=True), 1e-300))[inside[:self.T]]
            which = np.searchsorted(off[1:], np.nonzero(inside)[0], side="right") if self.G > 1 else np.zeros(inside.sum(), int)
            n = np.array([max(1, int((mask[off[g]:off[g + 1]] != 0).sum())) for g in range(self.G)])
            f = counts * self.E / (self.k * n[:, None])
            big = (self.gl * self.coef / n * f.max(1))[which][:, None] * np.nan_to_num(p)
            tol = 4 * ep * big + (U16 * np.abs(want) * 1.01 if self.tdt == torch.bfloat16 else 0) + 1e-37
            np.testing.assert_array_less(np.nan_to_num(np.abs(got - want)), np.nan_to_num(tol))


SIZES = [(1, 1, 1, 1), (1, 8, 2, 1), (16, 8, 2, 1), (7, 3, 2, 1), (40, 61, 4, 5), (300, 256, 8, 1), (129, 255, 16, 9),
         (2048, 64, 6, 1), (3001, 60, 4, 37), (5000, 7, 2, 3), (9000, 4, 1, 1), (2500, 128, 8, 700), (1500, 32, 8, 2),
         (700, 200, 3, 2), (40000, 2, 2, 5), (33000, 1, 1, 1), (1030, 100, 6, 1), (513, 252, 8, 3),
         (20000, 64, 2, 300), (4097, 129, 3, 512)]


@pytest.mark.parametrize("T,E,k,G", SIZES)
@pytest.mark.parametrize("dt,masked,pad", [("f32", False, 0), ("bf16", True, 4), ("f32", True, 3), ("bf16", False, 0)])
def test_sizes(T, E, k, G, dt, masked, pad):
    c = Case(T, E, k, G, dt, masked, pad)
    c.run()
    c.check()


@pytest.mark.parametrize("T,E,G", [(50, 16, 4), (6000, 16, 4)])
def test_rows_of_no_group_and_empty_groups(T, E, G):
    def tweak(c, x, rng):
        c.off = np.array([3, 3, T // 2, T // 2, T - 5], np.int32)
    c = Case(T, E, 2, G, masked=True, edge=3, tweak=tweak)
    c.run()
    c.check()
    assert float(c.out["loss"][0]) == 0 and float(c.out["loss"][2]) == 0


@pytest.mark.parametrize("T,G", [(40, 3), (9000, 3)])
def test_group_whose_mask_leaves_nothing(T, G):
    def tweak(c, x, rng):
        c.mask[c.off[1]:c.off[2]] = 0
        x[c.off[1]:c.off[2]] = np.nan        # dropped rows may hold anything
    c = Case(T, 8, 2, G, masked=True, tweak=tweak)
    c.run()
    c.check()
    assert float(c.out["loss"][1]) == 0
    assert (c.out["dlogits"][c.off[1]:c.off[2]] == 0).all()


@pytest.mark.parametrize("T", [30, 9000])
def test_infinite_and_extreme_logits(T):
    def tweak(c, x, rng):
        x[3, 2] = -np.inf
        x[4, :] = -np.inf
        x[5, :] = np.finfo(np.float32).min    # the type's lowest value throughout
        x[6, 1:] = np.finfo(np.float32).min
        x[7, :] *= 40.0
    c = Case(T, 8, 2, 1, tweak=tweak)
    c.run()
    off, mask = np.array([0, T]), np.ones(T, np.uint8)
    loss, counts, mean, d = balance(c.x64, c.idx, off, mask, c.coef, c.gl)
    got = c.out["dlogits"].double().cpu().numpy()
    assert (got[4] == 0).all() and got[3, 2] == 0
    # probabilities carry the rounding of arguments up to 300: 2 * (300 + 24) half steps
    tol = 4 * 2 * 324 * U32 * float(c.gl[0]) * c.coef / T * (counts.max() * 8 / (2 * T))
    assert np.abs(got - d).max() <= tol + 1e-37
    assert np.abs(c.out["mean_prob"].cpu().numpy() - mean).max() <= (2 * 324 + 872) * U32


@pytest.mark.parametrize("T", [30, 9000])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_nan_stays_in_its_row_and_group(T, bad):
    def tweak(c, x, rng):
        c.off = np.array([0, 10, T], np.int32)
        x[12, 3] = bad
    c = Case(T, 8, 2, 2, tweak=tweak)
    c.run()
    assert torch.isnan(c.out["dlogits"][12]).all()
    rest = torch.cat([c.out["dlogits"][:12], c.out["dlogits"][13:]])
    assert torch.isfinite(rest).all()
    assert torch.isfinite(c.out["loss"][0]) and torch.isnan(c.out["loss"][1])


@pytest.mark.parametrize("T", [33, 9000])
def test_indices_outside_are_not_counted(T):
    def tweak(c, x, rng):
        c.idx[::3, 0] = -1
        c.idx[1::5, 1] = 8
        c.idx[2::7, 1] = 2 ** 30
    c = Case(T, 8, 2, 1, tweak=tweak)
    c.run()
    c.check()


@pytest.mark.parametrize("T,E,G", [(48, 8, 3), (3000, 64, 3)])
def test_outputs_are_optional_and_the_same_bits(T, E, G):
    c = Case(T, E, 2, G, masked=True)
    full = {k: v.clone() for k, v in c.run().items()}
    for drop in ("loss", "counts", "mean_prob", "dlogits"):
        got = c.run(**{drop: None})
        for k, v in got.items():
            assert v is None or torch.equal(v, full[k]), (drop, k)


def test_no_tokens():
    c = Case(0, 8, 2, 1)
    c.run()
    assert float(c.out["loss"][0]) == 0 and (c.out["counts"] == 0).all() and (c.out["mean_prob"] == 0).all()
    assert (c.out["dlogits"] == 5).all()


@pytest.mark.parametrize("T,E,dt", [(40, 16, "f32"), (4000, 64, "bf16"), (4000, 61, "f32")])
def test_gradient_over_the_logits(T, E, dt):
    c = Case(T, E, 2, 2, dt)
    want = c.run()["dlogits"].clone()
    c.run(dlogits=c.logits)
    assert torch.equal(c.logits, want)


@pytest.mark.parametrize("T", [12, 8200])
def test_gradient_against_differences(T):
    """Central differences of the 64-bit loss with the counts held constant."""
    c = Case(T, 6, 2, 2)
    got = c.run()["dlogits"].double().cpu().numpy()
    one = np.ones(T, np.uint8)
    h = 1e-5
    for t, e in [(0, 0), (3, 5), (T - 1, 2)]:
        a, b = c.x64.copy(), c.x64.copy()
        a[t, e] += h
        b[t, e] -= h
        la, lb = (balance(x, c.idx, c.off, one, c.coef, c.gl)[0] for x in (a, b))
        want = float((c.gl * (la - lb)).sum()) / (2 * h)
        # third derivatives of a softmax are at most 1: h^2/6, and the difference's own rounding, 2^-52 of the loss / h
        scale = c.coef * c.gl.max() * 6 / max(1, min(np.diff(c.off)))
        assert abs(got[t, e] - want) <= scale * (h * h + 1e-5) + 4 * 2.0 ** -52 / h


def test_runs_give_the_same_bits_and_any_workspace_content():
    c = Case(20000, 64, 6, 11, masked=True)
    a = {k: v.clone() for k, v in c.run().items()}
    for _ in range(3):
        b = c.run()
        assert all(torch.equal(a[k], b[k]) for k in a)


def test_other_stream_and_graph():
    c = Case(5000, 32, 4, 3, masked=True)
    want = {k: v.clone() for k, v in c.run().items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.run(stream=side)
    assert all(torch.equal(got[k], want[k]) for k in want)
    with torch.cuda.stream(side):
        mira.mira_balance_loss(c.args)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mira.mira_balance_loss(c.args)
    for _ in range(4):
        for v in got.values():
            v.fill_(3)
        c.out["dlogits"].fill_(5.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], want[k]) for k in want)


def test_offsets_that_do_not_ascend_stay_inside():
    """Unspecified results, but no access outside the buffers."""
    for off in ([0, 50, 20, 9000], [-5, 100, 99999, 200], [9000, 0, 0, 0]):
        def tweak(c, x, rng):
            c.off = np.array(off, np.int32)
        for T in (60, 9000):
            c = Case(T, 8, 2, 3, tweak=tweak)
            c.run()
            assert (c.out["dlogits"].shape[0] == T)


@pytest.mark.parametrize("E", [2, 3, 5, 8])
@pytest.mark.parametrize("T,dt", [(37, "f32"), (20000, "f32"), (20000, "bf16")])
def test_all_experts_selected(E, T, dt):
    """Every expert selected by every token: f is 1 throughout and the gradient is
    zero but for roundings, which are those of the formula evaluated step by step
    in fp32 (elementwise, by torch)."""
    c = Case(T, E, E, 1, dt)
    got = c.run()["dlogits"][:T, :E]
    x = c.logits[:T, :E].float()
    e = torch.exp(x - x.amax(1, keepdim=True))
    p = e / e.sum(1, keepdim=True)
    n = torch.full((1,), float(T), device="cuda")
    f = torch.full((E,), float(T), device="cuda") * ((E * n) .reciprocal() * E)
    d = (c.dev["gl"] * c.coef / n) * p * (f - (f * p).sum(1, keepdim=True))
    # nothing larger than the roundings of w = sum f p (E + 3 of them) times the scale
    assert float(got.double().abs().max()) <= (E + 3) * 2 * U32 * float(c.gl[0]) * c.coef / T
    assert torch.equal(got, d.to(got.dtype))


@pytest.mark.parametrize("T,G", [(3000, 200), (30000, 200)])
def test_one_group_of_nearly_all_rows(T, G):
    """Both ways of sharing the work, with runs of empty groups on both sides."""
    def tweak(c, x, rng):
        c.off = np.concatenate([np.full(G // 2, 2), np.full(G // 2 - 10, T - 20), np.arange(T - 20, T + 1, 2)]).astype(np.int32)
        assert len(c.off) == G + 1
    c = Case(T, 64, 2, G, masked=True, tweak=tweak)
    c.run()
    c.check()


def test_two_streams_at_once():
    """Calls on their own workspaces and outputs, in flight together."""
    cases = [Case(T, 64, 4, G, seed=i) for i, (T, G) in enumerate(((20000, 1), (20000, 300), (300, 5)))]
    want = [{k: v.clone() for k, v in c.run().items()} for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(3):
        for c in cases:
            for v in c.out.values():
                v.fill_(3)
            c.out["dlogits"].fill_(5.0)
        torch.cuda.synchronize()
        for c, st in zip(cases, streams):
            mira.mira_balance_loss(c.args, st)
        torch.cuda.synchronize()
        for c, w in zip(cases, want):
            assert all(torch.equal(c.out[k], w[k]) for k in w)


# either side of each bound of the dispatch: one workgroup per group for all; counts by
# group; counts by chunks from zeros
@pytest.mark.parametrize("T,E,k,G,ran", [
    (512, 64, 4, 1, {"group"}), (513, 64, 4, 1, {"count", "rows"}), (16384, 64, 2, 1, {"count", "rows"}),
    (16385, 64, 2, 1, {"zero", "count", "rows"}), (2048, 64, 4, 16, {"group"}), (2049, 64, 4, 16, {"count", "rows", "finish"}),
    (21845, 64, 3, 16, {"count", "rows", "finish"}), (21846, 64, 3, 16, {"zero", "count", "rows", "finish"}),
    (32768, 32, 8, 64, {"count", "rows", "finish"}), (32769, 32, 8, 64, {"zero", "count", "rows", "finish"})])
def test_dispatch_bounds(T, E, k, G, ran):
    c = Case(T, E, k, G, masked=G > 1)
    mira.mira_profile_enable(True)
    mira.mira_profile_read()
    c.run()
    names = set(mira.mira_profile_read())
    mira.mira_profile_enable(False)
    assert names == {"balance_" + n for n in ran}
    c.check()


def _special(T, dt):
    low = float(torch.finfo(torch.float32 if dt == "f32" else torch.bfloat16).min)

    def tweak(c, x, rng):
        x[3, 2] = -np.inf
        x[4, :] = -np.inf
        x[5, :] = low                 # the type's lowest value throughout
        x[6, 1:] = low
        x[7, :] *= 40.0
        x[8, :], x[9, 1] = np.nan, np.inf   # dropped rows may hold anything
        x[10, :-1] = -np.inf          # one expert is left
        c.mask[:12] = 1
        c.mask[8] = c.mask[9] = 0
        c.idx[::3, 0] = -1            # not counted
        c.idx[1::5, 1] = c.E
        c.idx[2::7, 1] = 2 ** 30
    return tweak


def _check_special(T, E, k, dt):
    c = Case(T, E, k, 1, dt, masked=True, tweak=_special(T, dt))
    c.run()
    loss, counts, mean, d = balance(c.x64, c.idx, np.array([0, T]), c.mask, c.coef, c.gl)
    n = int((c.mask != 0).sum())
    assert np.array_equal(c.out["counts"].cpu().numpy(), counts)
    got = c.out["dlogits"].double().cpu().numpy()[:T]
    assert (got[[4, 8, 9]] == 0).all() and got[3, 2] == 0 and (got[10, :-1] == 0).all()
    # probabilities carry the rounding of arguments up to 300 (below, exp is 0): 2 * (300 + 24) half steps
    tol = 4 * 2 * 324 * U32 * float(c.gl[0]) * c.coef / n * (counts.max() * E / (k * n))
    assert (np.abs(got - d) <= tol + (1.01 * U16 * np.abs(d) if dt == "bf16" else 0) + 1e-37).all()
    assert np.abs(c.out["mean_prob"].cpu().numpy() - mean).max() <= (2 * 324 + 872) * U32
    assert abs(float(c.out["loss"][0]) - loss[0]) <= (2 * 324 + 872 + 300) * U32 * loss[0]


# the special values of the tests above where a router is larger than they have it, each
# width of its row's lanes
@pytest.mark.parametrize("E", [9, 16, 17, 61, 64, 100, 256])
@pytest.mark.parametrize("T", [30, 9000])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_special_logits_of_larger_routers(E, T, dt):
    _check_special(T, E, 2, dt)


# and of few experts, some of them selected and all
@pytest.mark.parametrize("E,k", [(3, 2), (3, 3), (5, 2), (5, 5), (8, 7), (8, 8), (8, 16), (12, 12)])
@pytest.mark.parametrize("T", [30, 9000])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_special_logits_of_few_experts(E, k, T, dt):
    _check_special(T, E, k, dt)


@pytest.mark.parametrize("T", [30, 9000])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_nan_stays_in_its_row_and_group_of_all_selected(T, bad):
    def tweak(c, x, rng):
        c.off = np.array([0, 10, T], np.int32)
        x[12, 3] = bad
    c = Case(T, 8, 8, 2, tweak=tweak)
    c.run()
    assert torch.isnan(c.out["dlogits"][12]).all()
    assert torch.isfinite(torch.cat([c.out["dlogits"][:12], c.out["dlogits"][13:]])).all()
    assert torch.isfinite(c.out["loss"][0]) and torch.isnan(c.out["loss"][1])


@pytest.mark.parametrize("E", [9, 16, 64, 250])
@pytest.mark.parametrize("T", [30, 9000])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_nan_stays_in_its_row_and_group_of_larger_routers(E, T, bad):
    def tweak(c, x, rng):
        c.off = np.array([0, 10, T], np.int32)
        x[12, 3] = bad
    c = Case(T, E, 2, 2, tweak=tweak)
    c.run()
    assert torch.isnan(c.out["dlogits"][12]).all()
    assert torch.isfinite(torch.cat([c.out["dlogits"][:12], c.out["dlogits"][13:]])).all()
    assert torch.isfinite(c.out["loss"][0]) and torch.isnan(c.out["loss"][1])


@pytest.mark.parametrize("off", [[0, 50, 20, 9000], [-5, 100, 99999, 200], [9000, 0, 0, 0], [0, 9000, 0, 9000], [20, 10, 10, 5]])
@pytest.mark.parametrize("T,E", [(60, 8), (60, 64), (9000, 8), (9000, 64), (30000, 8), (30000, 61)])
def test_offsets_that_do_not_ascend_write_only_their_buffers(T, E, off):
    """Every buffer in the middle of a larger one; each way of counting."""
    def tweak(c, x, rng):
        c.off = np.array(off, np.int32)
    c = Case(T, E, 2, 3, masked=True, tweak=tweak)
    c.run()
    want = {"small": T == 60, "zero": T == 30000}
    G, pad = 3, 1024
    sizes = dict(loss=G, counts=G * E, mean_prob=G * E, dlogits=T * E)
    flat = {k: torch.full((n + 2 * pad,), 77, dtype=torch.int32 if k == "counts" else torch.float32, device="cuda") for k, n in sizes.items()}
    for k, v in flat.items():
        setattr(c.args, k, v[pad:])
    ws = torch.full((c.args.workspace_bytes + 2 * pad,), 0xA5, dtype=torch.uint8, device="cuda")
    c.args.workspace = ws[pad:]
    mira.mira_profile_enable(True)
    mira.mira_profile_read()
    mira.mira_balance_loss(c.args)
    torch.cuda.synchronize()
    ran = set(mira.mira_profile_read())
    mira.mira_profile_enable(False)
    assert ("balance_group" in ran) == want["small"] and ("balance_zero" in ran) == want["zero"], ran
    for k, v in flat.items():
        assert (v[:pad] == 77).all() and (v[pad + sizes[k]:] == 77).all(), k
    assert (ws[:pad] == 0xA5).all() and (ws[pad + c.args.workspace_bytes:] == 0xA5).all()


def _in_order(v):
    """Sum over the last axis as the kernel's lanes take it: the largest power of two of
    lanes, a second value added to a lane's first, then pairs, pairs of pairs and so on."""
    E = v.shape[1]
    L = 1 << (E.bit_length() - 1)
    s = v[:, :L].clone()
    s[:, :E - L] = s[:, :E - L] + v[:, L:]
    while s.shape[1] > 1:
        s = s[:, 0::2] + s[:, 1::2]
    return s


@pytest.mark.parametrize("E", range(1, 17))
@pytest.mark.parametrize("T,k,dt", [(37, 0, "f32"), (20000, 0, "f32"), (20000, 0, "bf16"), (20000, 16, "f32")])
def test_all_experts_selected_up_to_sixteen(E, T, k, dt):
    """As many selected as there are experts, or more (some twice).  The gradient of equal
    counts is zero but for roundings; up to 8 experts each step of the formula is rounded
    once in fp32."""
    c = Case(T, E, k or E, 1, dt)
    got = c.run()["dlogits"][:T, :E]
    c.check()
    x = c.logits[:T, :E].float()
    e = torch.exp(x - x.amax(1, keepdim=True))
    p = e / _in_order(e)
    n = torch.full((1,), float(T), device="cuda")
    f = c.out["counts"].float() * ((c.k * n).reciprocal() * E)
    d = (c.dev["gl"] * c.coef / n) * p * (f - _in_order(f * p))
    if not k:  # the sums of e and of f e have 6 roundings each at most, the steps between 3: fewer than these
        assert float(got.double().abs().max()) <= 24 * U32 * float(c.gl[0]) * c.coef / T
    assert E > 8 or torch.equal(got, d.to(got.dtype))


@pytest.mark.parametrize("E,k", [(2, 1), (3, 2), (5, 4), (7, 6), (8, 7), (9, 8), (16, 15), (17, 16)])
@pytest.mark.parametrize("T,dt,masked", [(37, "f32", True), (20000, "f32", False), (20000, "bf16", True)])
def test_all_experts_but_one_selected(E, k, T, dt, masked):
    c = Case(T, E, k, 3, dt, masked)
    c.run()
    c.check()
