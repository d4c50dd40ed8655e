"""Workloads of the operators that complete an expert layer around the 8-bit
products, forward and backward: the root-mean-square norm with the residual's
addition and an 8-bit output, the selection of experts from their scores with
the order of the (token, expert) pairs, the weighted combine of the pairs'
rows, and the gradient of SwiGLU in 8 bits.

listed() gives the named cases, draw() more of the same ranges; prepare() makes
what a program holds before the call, run() is one pass (in elementary torch
operations, or through the library where `own` is true), exact() the same
outputs in 64-bit torch."""
import math

import numpy as np
import torch

own = False

BLOCK = 128       # columns that share a scale
E4M3_MAX = 448.0
Q_EPS = 1e-8      # the smallest block maximum, as in this repository's expert packer
NORM_EPS = 1e-6
TINY = 1e-20      # beside the sum of the selected scores

MOST_NORM = 16384 * 4096         # values of a drawn norm
MOST_LOGITS = 131072 * 256       # of a drawn selection
MOST_PAIR_VALUES = 4096 * 3 * 4096  # of a drawn combine: pairs and tokens times columns
MOST_SWIGLU = 8192 * 14336       # of a drawn SwiGLU gradient in bf16 to e4m3, fewer of wider types


def listed():
    return [
        # a decode step's token before the experts: residual added, bf16 for the router, e4m3 for the products
        dict(name="norm_token_1", op="norm", rows=1, cols=4096, dt="bf16", res=True, y=True, q=True),
        # a prompt
        dict(name="norm_prompt_4096", op="norm", rows=4096, cols=4096, dt="bf16", res=True, y=True, q=True),
        # odd sizes, fp32, the gradient with the weight's
        dict(name="norm_grad_odd_1201", op="norm_grad", rows=1201, cols=2001, dt="f32", res=False),
        # the tokens of a training step, with the residual stream's own gradient
        dict(name="norm_grad_16384", op="norm_grad", rows=16384, cols=4096, dt="bf16", res=True),
        # a decode step of sixteen tokens through an 8-expert router: softmax, renormalised
        dict(name="route_step_16", op="route", T=16, E=8, k=2, S=0, score="softmax", bias=False, groups=1, top_groups=1, best=1,
             renorm=True, masked=False, dt="f32"),
        # a large batch through the widest router: sigmoid scores, a balancing bias, four groups of eight kept
        dict(name="route_long_131072", op="route", T=131072, E=256, k=8, S=0, score="sigmoid", bias=True, groups=8, top_groups=4, best=2,
             renorm=True, masked=False, dt="f32"),
        # the gradient of a packed, padded batch's weights, on top of the balance loss's, bf16 and odd sizes
        dict(name="route_grad_30011", op="route_grad", T=30011, E=61, k=4, score="softmax", renorm=False, masked=True, add=True, dt="bf16"),
        # sixteen tokens of a fine-grained layer, two shared experts, fp32 rows from the down product
        dict(name="combine_step_16", op="combine", T=16, k=6, S=2, cols=2048, ydt="f32", dt="bf16", res=True, weights=True),
        # a prompt through a two-expert layer
        dict(name="combine_prompt_4096", op="combine", T=4096, k=2, S=0, cols=4096, ydt="bf16", dt="bf16", res=True, weights=True),
        # the gradient of a fine-grained prompt: weights' in fp32, rows' in e4m3 for the next product
        dict(name="combine_grad_2048", op="combine_grad", T=2048, k=6, S=2, cols=2048, ydt="bf16", dt="bf16", dy=False, q=True),
        # odd sizes, fp32 throughout
        dict(name="swiglu_grad_301", op="swiglu_grad", rows=301, cols=1001, dt="f32", dx=True, q=False),
        # the largest: between the two products of a training step's backward pass
        dict(name="swiglu_grad_8192", op="swiglu_grad", rows=8192, cols=14336, dt="bf16", dx=False, q=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "route", "route", "route_grad", "combine", "combine_grad", "swiglu_grad"])
    dt = rng.choice(["f32", "bf16", "bf16"])
    if op in ("norm", "norm_grad", "swiglu_grad"):
        while True:
            rows, cols = _log_int(rng, 1, 65536), _log_int(rng, 64, 16384)
            if rows * cols <= (MOST_SWIGLU * 2 // 3 if op == "swiglu_grad" else MOST_NORM) // (2 if dt == "f32" else 1):
                break
        outs = rng.choice([(True, False), (False, True), (True, True)])
        if op == "norm":
            return dict(op=op, rows=rows, cols=cols, dt=dt, res=rng.random() < 0.7, y=outs[0], q=outs[1])
        if op == "norm_grad":
            return dict(op=op, rows=rows, cols=cols, dt=dt, res=rng.random() < 0.7)
        return dict(op=op, rows=rows, cols=cols, dt=dt, dx=outs[0], q=outs[1])
    if op in ("route", "route_grad"):
        while True:
            T, E = _log_int(rng, 1, 131072), _log_int(rng, 2, 256)
            if T * E <= MOST_LOGITS:
                break
        score, renorm, masked = rng.choice(["softmax", "sigmoid"]), rng.random() < 0.6, rng.random() < 0.3
        if op == "route_grad":
            return dict(op=op, T=T, E=E, k=rng.randint(1, min(8, E)), score=score, renorm=renorm, masked=masked, add=rng.random() < 0.4, dt=dt)
        groups = rng.choice([1, 1, *(g for g in range(2, 33) if E % g == 0)])
        kept = rng.randint(1, groups)
        S = rng.choice([0, 0, 1, 2])
        return dict(op=op, T=T, E=E - S if groups == 1 and E > 8 else E, k=rng.randint(1, min(8, kept * (E // groups), max(1, E - S))),
                    S=S if groups == 1 and E > 8 else 0, score=score, bias=rng.random() < 0.5, groups=groups, top_groups=kept,
                    best=rng.randint(1, min(2, E // groups)), renorm=renorm, masked=masked, dt=dt)
    ydt = rng.choice(["f32", "bf16"])
    while True:
        T, k, S, cols = _log_int(rng, 1, 32768), rng.randint(1, 8), rng.choice([0, 0, 1, 2]), _log_int(rng, 64, 16384)
        if T * (k + S + 1) * cols <= MOST_PAIR_VALUES:
            break
    if op == "combine":
        return dict(op=op, T=T, k=k, S=S, cols=cols, ydt=ydt, dt=dt, res=rng.random() < 0.5, weights=rng.random() < 0.8)
    dy, q = rng.choice([(True, False), (False, True), (True, True)])
    return dict(op=op, T=T, k=k, S=S, cols=cols, ydt=ydt, dt=dt, dy=dy, q=q)


# ---- inputs -----------------------------------------------------------------

def _gen(seed, *more):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(np.random.SeedSequence([seed, *more]).generate_state(1, np.uint64)[0] >> np.uint64(1)))
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _rand(g, *shape):
    return torch.rand(shape, generator=g, device="cuda", dtype=torch.float32)


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _blocks(n):
    return -(-n // BLOCK)


def _pad16(n):
    return -(-n // 16) * 16


def _activations(g, rows, cols):
    """A few channels of activations are much larger than the others."""
    x = _randn(g, rows, cols)
    x[:, torch.randperm(cols, generator=g, device="cuda")[: max(1, cols // 256)]] *= 20.0
    return x


def _prepare_norm(c, seed):
    g, dt = _gen(seed, 11), _dtype(c["dt"])
    s = dict(c=c, x=_activations(g, c["rows"], c["cols"]).to(dt), residual=None, w=(1.0 + 0.1 * _randn(g, c["cols"])).to(dt))
    if c["res"]:
        s["residual"] = (3.0 * _randn(g, c["rows"], c["cols"])).to(dt)
    return s


def _prepare_norm_grad(c, seed):
    g, dt = _gen(seed, 12), _dtype(c["dt"])
    s = dict(c=c, h=_activations(g, c["rows"], c["cols"]).to(dt), dy=(0.01 * _randn(g, c["rows"], c["cols"])).to(dt), dsum=None,
             w=(1.0 + 0.1 * _randn(g, c["cols"])).to(dt))
    if c["res"]:
        s["dsum"] = (0.01 * _randn(g, c["rows"], c["cols"])).to(dt)
    return s


def _logits(g, T, E):
    return _randn(g, T, E) * 1.5 - 0.5 * torch.log(torch.arange(1, E + 1, device="cuda", dtype=torch.float32))


def _mask(c, g):
    return (_rand(g, c["T"]) < 0.9).to(torch.uint8) if c["masked"] else None


def _prepare_route(c, seed):
    g = _gen(seed, 13)
    return dict(c=c, logits=_logits(g, c["T"], c["E"]).to(_dtype(c["dt"])), bias=0.1 * _randn(g, c["E"]) if c["bias"] else None,
                mask=_mask(c, g), scale=2.5 if c["score"] == "sigmoid" else 1.0)


def _prepare_route_grad(c, seed):
    g, dt = _gen(seed, 14), _dtype(c["dt"])
    logits = _logits(g, c["T"], c["E"]).to(dt)
    idx = logits.float().topk(c["k"], dim=1).indices.to(torch.int32)
    mask = _mask(c, g)
    if mask is not None:
        idx[mask == 0] = -1
    return dict(c=c, logits=logits, idx=idx.contiguous(), dweight=0.01 * _randn(g, c["T"], c["k"]),
                add=(1e-4 * _randn(g, c["T"], c["E"])).to(dt) if c["add"] else None, scale=2.5 if c["score"] == "sigmoid" else 1.0)


def _positions(g, c):
    """Positions of the pairs in the experts' order, as a skewed router of 16 experts gives them."""
    T, k, S = c["T"], c["k"], c["S"]
    expert = (_randn(g, T, 16) - 0.5 * torch.log(torch.arange(1, 17, device="cuda", dtype=torch.float32))).topk(k, dim=1).indices
    group = torch.cat([expert.reshape(-1), torch.arange(16, 16 + S, device="cuda").repeat_interleave(T)])
    order = torch.sort(group, stable=True).indices
    pos = torch.empty_like(order)
    pos[order] = torch.arange(order.numel(), device="cuda")
    return pos.to(torch.int32)


def _prepare_combine(c, seed):
    g = _gen(seed, 15)
    T, k, S, cols = c["T"], c["k"], c["S"], c["cols"]
    s = dict(c=c, pos=_positions(g, c), w=torch.softmax(_randn(g, T, k), 1))
    s["y"] = _randn(g, T * (k + S), cols).to(_dtype(c["ydt"]))
    if c["op"] == "combine":
        s["residual"] = _randn(g, T, cols).to(_dtype(c["dt"])) if c["res"] else None
        s["w"] = s["w"] if c["weights"] else None
    else:
        s["dout"] = (0.01 * _activations(g, T, cols)).to(_dtype(c["dt"]))
    return s


def _prepare_swiglu_grad(c, seed):
    g, dt = _gen(seed, 16), _dtype(c["dt"])
    return dict(c=c, x=_activations(g, c["rows"], 2 * c["cols"]).to(dt), dact=(0.01 * _randn(g, c["rows"], c["cols"])).to(dt))


def prepare(case, seed):
    make = dict(norm=_prepare_norm, norm_grad=_prepare_norm_grad, route=_prepare_route, route_grad=_prepare_route_grad,
                combine=_prepare_combine, combine_grad=_prepare_combine, swiglu_grad=_prepare_swiglu_grad)
    return make[case["op"]](case, seed)


# ---- the plain forms ----------------------------------------------------------

def _quant(x):
    """e4m3 values and scales of each block of 1 x 128 of fp32 rows."""
    rows, cols = x.shape
    nc = _blocks(cols)
    v = torch.nn.functional.pad(x, (0, nc * BLOCK - cols)).view(rows, nc, BLOCK)
    a = v.abs().amax(2).clamp(min=Q_EPS)
    top = torch.full_like(a, E4M3_MAX)  # tensor by tensor: a division by a number multiplies by its rounded inverse
    q = (v * (top / a)[:, :, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return q.view(rows, nc * BLOCK)[:, :cols].contiguous(), a / top


def _norm(s):
    c, dt = s["c"], _dtype(s["c"]["dt"])
    out = {}
    h = s["x"].float()
    if s["residual"] is not None:
        out["sum"] = (h + s["residual"].float()).to(dt)
        h = out["sum"].float()
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + NORM_EPS) * s["w"].float()
    if c["y"]:
        out["y"] = y.to(dt)
    if c["q"]:
        out["q"], out["scale"] = _quant(y)
    return out


def _norm_grad(s):
    h, dy = s["h"].float(), s["dy"].float()
    r = torch.rsqrt((h * h).mean(1, keepdim=True) + NORM_EPS)
    g = dy * s["w"].float()
    dx = r * (g - h * (r * r * (g * h).mean(1, keepdim=True)))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    return dict(dx=dx.to(s["h"].dtype), dweight=(dy * h * r).sum(0))


def _scores(x, score):
    if score == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-x))
    e = torch.exp(x - x.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _weights(sel, c, scale):
    return sel * (scale / (sel.sum(1, keepdim=True) + TINY)) if c["renorm"] else sel * scale


def _route(s):
    c = s["c"]
    T, E, k, S, n = c["T"], c["E"], c["k"], c["S"], c["groups"]
    # the selection in 64 bits: neighbours at its border are closer than 32 tell apart
    wide = _scores(s["logits"].double(), c["score"])
    choice = wide if s["bias"] is None else wide + s["bias"].double()
    if n > 1:
        best = choice.view(T, n, E // n).topk(c["best"], dim=2).values.sum(2)
        kept = torch.sort(best, dim=1, descending=True, stable=True).indices[:, : c["top_groups"]]
        keep = torch.zeros(T, n, dtype=torch.bool, device="cuda").scatter_(1, kept, True)
        choice = choice.masked_fill(~keep.repeat_interleave(E // n, 1), -math.inf)
    idx = torch.sort(choice, dim=1, descending=True, stable=True).indices[:, :k]
    weight = _weights(_scores(s["logits"].float(), c["score"]).gather(1, idx), c, s["scale"])
    group = torch.cat([idx.reshape(-1), torch.arange(E, E + S, device="cuda").repeat_interleave(T)])
    if s["mask"] is not None:
        drop = s["mask"] == 0
        idx, weight = idx.masked_fill(drop[:, None], -1), weight.masked_fill(drop[:, None], 0.0)
        group = group.masked_fill(torch.cat([drop.repeat_interleave(k), drop.repeat(S)]), E + S)
    counts = torch.zeros(E + S + 1, dtype=torch.int64, device="cuda").scatter_add_(0, group, torch.ones_like(group))
    offsets = torch.nn.functional.pad(counts[: E + S].cumsum(0), (1, 0))
    order = torch.sort(group, stable=True).indices
    place = torch.arange(group.numel(), device="cuda")
    valid = place < offsets[-1]
    pos = torch.empty_like(place).scatter_(0, order, place.masked_fill(~valid, -1))
    i32 = torch.int32
    return dict(idx=idx.to(i32), weight=weight, counts=counts[: E + S].to(i32), offsets=offsets.to(i32),
                order=order.masked_fill(~valid, -1).to(i32), pos=pos.to(i32))


def _route_grad(s):
    c, x = s["c"], s["logits"].float()
    has = s["idx"] >= 0
    idx = s["idx"].clamp(min=0).long()
    p = _scores(x, c["score"])
    sel, g = p.gather(1, idx) * has, s["dweight"] * has
    if c["renorm"]:
        total = sel.sum(1, keepdim=True) + TINY
        mean = (g * sel).sum(1, keepdim=True) / total
        ds, rest = s["scale"] * (g - mean) / total * has, s["scale"] * mean * (TINY / total)
    else:
        ds, rest = s["scale"] * g, s["scale"] * (g * sel).sum(1, keepdim=True)
    ds = torch.zeros_like(p).scatter_add_(1, idx, ds)
    d = ds * p * _scores(-x, "sigmoid") if c["score"] == "sigmoid" else p * (ds - rest)
    if s["add"] is not None:
        d = d + s["add"].float()
    return dict(dlogits=d.to(s["logits"].dtype))


def _pairs_of(s):
    """Positions [T][k + S] of each token's pairs."""
    c = s["c"]
    n = c["T"] * c["k"]
    return torch.cat([s["pos"][:n].view(c["T"], c["k"]), s["pos"][n:].view(c["S"], c["T"]).t()], 1).long()


def _pair_weights(s):
    c = s["c"]
    w = torch.ones(c["T"], c["k"], device="cuda") if s["w"] is None else s["w"]
    return torch.nn.functional.pad(w, (0, c["S"]), value=1.0)


def _combine(s):
    out = (s["y"][_pairs_of(s)].float() * _pair_weights(s)[:, :, None]).sum(1)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return dict(out=out.to(_dtype(s["c"]["dt"])))


def _combine_grad(s):
    c = s["c"]
    at, d = _pairs_of(s), s["dout"].float()
    out = dict(dweight=(s["y"][at[:, : c["k"]]].float() * d[:, None, :]).sum(2))
    rows = torch.empty(s["y"].shape, device="cuda")
    rows[at.reshape(-1)] = (d[:, None, :] * _pair_weights(s)[:, :, None]).view(-1, c["cols"])
    if c["dy"]:
        out["dy"] = rows.to(s["y"].dtype)
    if c["q"]:
        out["q"], out["scale"] = _quant(rows)
    return out


def _swiglu_grad(s):
    c, x, d = s["c"], s["x"].float(), s["dact"].float()
    gate, up = x[:, : c["cols"]], x[:, c["cols"]:]
    sig, rest = 1.0 / (1.0 + torch.exp(-gate)), 1.0 / (1.0 + torch.exp(gate))
    dx = torch.cat([d * up * sig * (1.0 + gate * rest), d * gate * sig], 1)
    out = {}
    if c["dx"]:
        out["dx"] = dx.to(s["x"].dtype)
    if c["q"]:
        out["q"], out["scale"] = _quant(dx)
    return out


# ---- the library's calls --------------------------------------------------------

def _plan(s):
    """Outputs, workspace and arguments that a program keeps from call to call."""
    import paper_2609_38090_amd as mira
    c, op = s["c"], s["c"]["op"]
    code = {"f32": mira.MIRA_F32, "bf16": mira.MIRA_BF16}
    new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    out, held = {}, {}

    def eight_bits(rows, cols):
        held["q"], held["scale"] = new(rows, _pad16(cols), dtype=torch.float8_e4m3fn), new(rows, _blocks(cols))
        out["q"], out["scale"] = held["q"][:, :cols], held["scale"]

    if op == "norm":
        rows, cols, dt = c["rows"], c["cols"], _dtype(c["dt"])
        if c["res"]:
            held["sum"] = out["sum"] = new(rows, cols, dtype=dt)
        if c["y"]:
            held["y"] = out["y"] = new(rows, cols, dtype=dt)
        if c["q"]:
            eight_bits(rows, cols)
        t = code[c["dt"]]
        args = mira.RmsNormArgs(x=s["x"], residual=s["residual"], weight=s["w"], x_dtype=t, w_dtype=t, y_dtype=t, rows=rows, cols=cols,
                                eps=NORM_EPS, q_eps=Q_EPS, **held)
        return mira.mira_rmsnorm, args, out
    if op == "norm_grad":
        rows, cols, t = c["rows"], c["cols"], code[c["dt"]]
        out = dict(dx=new(rows, cols, dtype=_dtype(c["dt"])), dweight=new(cols))
        nb = mira.mira_rmsnorm_grad_workspace_bytes(rows, cols)
        args = mira.RmsNormGradArgs(dy=s["dy"], dsum=s["dsum"], h=s["h"], weight=s["w"], x_dtype=t, w_dtype=t, y_dtype=t, rows=rows, cols=cols,
                                    eps=NORM_EPS, workspace=new(nb, dtype=torch.uint8), workspace_bytes=nb, **out)
        return mira.mira_rmsnorm_grad, args, out
    if op in ("route", "route_grad"):
        T, E, k = c["T"], c["E"], c["k"]
        flags = (mira.MIRA_ROUTE_SIGMOID if c["score"] == "sigmoid" else 0) | (mira.MIRA_ROUTE_RENORM if c["renorm"] else 0)
        if op == "route_grad":
            out = dict(dlogits=new(T, E, dtype=_dtype(c["dt"])))
            args = mira.RouteSelectGradArgs(logits=s["logits"], topk_idx=s["idx"], dweight=s["dweight"], add=s["add"], logits_dtype=code[c["dt"]],
                                            n_tokens=T, n_experts=E, top_k=k, flags=flags, scale=s["scale"], **out)
            return mira.mira_route_select_grad, args, out
        S = c["S"]
        out = dict(idx=i32(T, k), weight=new(T, k), counts=i32(E + S), offsets=i32(E + S + 1), order=i32(T * (k + S)), pos=i32(T * (k + S)))
        nb = mira.mira_route_select_workspace_bytes(T, E, k, S)
        args = mira.RouteSelectArgs(logits=s["logits"], bias=s["bias"], mask=s["mask"], logits_dtype=code[c["dt"]], n_tokens=T, n_experts=E,
                                    top_k=k, n_shared=S, n_groups=c["groups"], top_groups=c["top_groups"], group_best=c["best"], flags=flags,
                                    scale=s["scale"], topk_idx=out["idx"], topk_weight=out["weight"], expert_counts=out["counts"],
                                    expert_offsets=out["offsets"], pair_order=out["order"], pair_pos=out["pos"],
                                    workspace=new(nb, dtype=torch.uint8), workspace_bytes=nb)
        return mira.mira_route_select, args, out
    if op == "combine":
        out = dict(out=new(c["T"], c["cols"], dtype=_dtype(c["dt"])))
        args = mira.CombineArgs(y=s["y"], topk_weight=s["w"], pair_pos=s["pos"], residual=s["residual"], n_tokens=c["T"], top_k=c["k"],
                                n_shared=c["S"], cols=c["cols"], y_rows=s["y"].shape[0], y_dtype=code[c["ydt"]], out_dtype=code[c["dt"]], **out)
        return mira.mira_combine, args, out
    if op == "combine_grad":
        if c["dy"]:
            held["dy"] = out["dy"] = new(*s["y"].shape, dtype=s["y"].dtype)
        if c["q"]:
            eight_bits(*s["y"].shape)
        held["dweight"] = out["dweight"] = new(c["T"], c["k"])
        args = mira.CombineGradArgs(dout=s["dout"], y=s["y"], topk_weight=s["w"], pair_pos=s["pos"], n_tokens=c["T"], top_k=c["k"],
                                    n_shared=c["S"], cols=c["cols"], y_rows=s["y"].shape[0], y_dtype=code[c["ydt"]], out_dtype=code[c["dt"]],
                                    q_eps=Q_EPS, **held)
        return mira.mira_combine_grad, args, out
    rows, cols, t = c["rows"], c["cols"], code[c["dt"]]
    if c["dx"]:
        held["dx"] = out["dx"] = new(rows, 2 * cols, dtype=_dtype(c["dt"]))
    if c["q"]:
        eight_bits(rows, 2 * cols)
    args = mira.SwigluGradArgs(x=s["x"], dact=s["dact"], x_dtype=t, d_dtype=t, rows=rows, cols=cols, q_eps=Q_EPS, **held)
    return mira.mira_swiglu_grad, args, out


def run(state):
    if own:
        if "plan" not in state:
            state["plan"] = _plan(state)
        call, args, out = state["plan"]
        call(args)
        return out
    form = dict(norm=_norm, norm_grad=_norm_grad, route=_route, route_grad=_route_grad, combine=_combine, combine_grad=_combine_grad,
                swiglu_grad=_swiglu_grad)
    return form[state["c"]["op"]](state)


def work(case):
    c, op = case, case["op"]
    w = 4 if c["dt"] == "f32" else 2
    if op in ("norm", "norm_grad", "swiglu_grad"):
        n = c["rows"] * c["cols"]
        scales = 4 * c["rows"] * _blocks(c["cols"])
        if op == "norm":
            return dict(bytes=n * w * (1 + 2 * c["res"] + c["y"]) + c["q"] * (n + scales) + c["cols"] * w, flops=(6 + 3 * c["q"]) * n)
        if op == "norm_grad":
            return dict(bytes=n * w * (3 + c["res"]) + c["cols"] * (w + 4), flops=12 * n)
        return dict(bytes=n * w * (3 + 2 * c["dx"]) + c["q"] * 2 * (n + scales), flops=(14 + 6 * c["q"]) * n)
    T, k = c["T"], c["k"]
    if op == "route":
        pairs = T * (k + c["S"])
        return dict(bytes=T * c["E"] * w + 8 * T * k + 8 * pairs + 8 * (c["E"] + c["S"]) + (4 * c["E"] if c["bias"] else 0) + (T if c["masked"] else 0),
                    flops=8 * T * c["E"])
    if op == "route_grad":
        # sigmoid scores need the selected logits only
        read = c["E"] if c["score"] == "softmax" else k
        return dict(bytes=T * w * (read + c["E"] * (1 + c["add"])) + 8 * T * k, flops=8 * T * (c["E"] if c["score"] == "softmax" else k))
    yw, pairs = 4 if c["ydt"] == "f32" else 2, T * (k + c["S"])
    if op == "combine":
        return dict(bytes=pairs * (c["cols"] * yw + 4) + T * c["cols"] * w * (1 + c["res"]) + (4 * T * k if c["weights"] else 0),
                    flops=2 * pairs * c["cols"])
    return dict(bytes=T * k * c["cols"] * yw + T * c["cols"] * w + pairs * (4 + c["cols"] * yw * c["dy"] + c["q"] * (c["cols"] + 4 * _blocks(c["cols"])))
                + 8 * T * k, flops=(3 + 3 * c["q"]) * pairs * c["cols"])


# ---- the definitions in 64 bits ---------------------------------------------------

def _to_e4m3(v):
    """64-bit values rounded to the nearest e4m3 value, ties to even."""
    e = torch.frexp(v.abs().clamp(min=2.0 ** -6))[1] - 1
    step = torch.ldexp(torch.ones_like(v), e - 3)
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _exact_quant(x):
    rows, cols = x.shape
    nc = _blocks(cols)
    full = torch.zeros(rows, nc * BLOCK, dtype=torch.float64, device="cuda")
    full[:, :cols] = x
    v = full.view(rows, nc, BLOCK)
    a = v.abs().amax(2).clamp(min=Q_EPS)
    inverse = (E4M3_MAX / a).float().double()  # held in 32 bits by definition
    return _to_e4m3(v * inverse[:, :, None]).view_as(full)[:, :cols].contiguous(), a / E4M3_MAX


def _exact_norm(s):
    c, out = s["c"], {}
    h = s["x"].double()
    if s["residual"] is not None:
        out["sum"] = (h + s["residual"].double()).to(s["x"].dtype).double()  # the norm is of the sum as it is held
        h = out["sum"]
    y = h / torch.sqrt(h.pow(2).sum(1, keepdim=True) / c["cols"] + NORM_EPS) * s["w"].double()
    if c["y"]:
        out["y"] = y
    if c["q"]:
        out["q"], out["scale"] = _exact_quant(y)
    return out


def _exact_norm_grad(s):
    h, dy, w, n = s["h"].double(), s["dy"].double(), s["w"].double(), s["c"]["cols"]
    v = h.pow(2).sum(1) / n + NORM_EPS
    inner = (h * dy) @ w  # of y = h v^-1/2 w: dy w v^-1/2 - h v^-3/2 (h . dy w) / n
    dx = dy * w / v.sqrt()[:, None] - h * (inner / n / (v * v.sqrt()))[:, None]
    if s["dsum"] is not None:
        dx += s["dsum"].double()
    return dict(dx=dx, dweight=(dy * h / v.sqrt()[:, None]).sum(0))


def _exact_scores(s):
    x = s["logits"].double()
    return torch.softmax(x, 1) if s["c"]["score"] == "softmax" else torch.sigmoid(x)


def _take_best(v, times):
    """The largest of each row, `times` times over: lowest index first among equals."""
    v, got = v.clone(), []
    at = torch.arange(v.shape[1], device="cuda").expand_as(v)
    for _ in range(times):
        got.append(torch.where(v == v.amax(1, keepdim=True), at, v.shape[1]).amin(1))
        v.scatter_(1, got[-1][:, None], -math.inf)
    return torch.stack(got, 1)


def _exact_route(s):
    c = s["c"]
    T, E, k, S, n = c["T"], c["E"], c["k"], c["S"], c["groups"]
    p = _exact_scores(s)
    choice = p.clone() if s["bias"] is None else p + s["bias"].double()
    if n > 1:
        size = E // n
        of_group = torch.stack([choice[:, g * size:(g + 1) * size].sort(1).values[:, size - c["best"]:].sum(1) for g in range(n)], 1)
        kept = _take_best(of_group, c["top_groups"])
        for g in range(n):
            choice[(kept != g).all(1), g * size:(g + 1) * size] = -math.inf
    idx = _take_best(choice, k)
    w = p.gather(1, idx)
    w = w * s["scale"] / (w.sum(1, keepdim=True) + TINY) if c["renorm"] else w * s["scale"]
    if s["mask"] is not None:
        w[s["mask"] == 0], idx[s["mask"] == 0] = 0.0, -1
    kept = torch.ones(T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"].bool()
    flat, tokens = idx.reshape(-1), kept.nonzero()[:, 0]
    lists = [(flat == e).nonzero()[:, 0] for e in range(E)] + [T * k + x * T + tokens for x in range(S)]
    counts = torch.tensor([len(x) for x in lists], dtype=torch.int32, device="cuda")
    order, pos = (torch.full((T * (k + S),), -1, dtype=torch.int32, device="cuda") for _ in range(2))
    pairs = torch.cat(lists)
    order[: len(pairs)] = pairs.to(torch.int32)
    pos[pairs] = torch.arange(len(pairs), dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, *np.cumsum(counts.tolist())], dtype=torch.int32, device="cuda")
    return dict(idx=idx.to(torch.int32), weight=w, counts=counts, offsets=offsets, order=order, pos=pos)


def _exact_route_grad(s):
    c, p, g = s["c"], _exact_scores(s), s["dweight"].double()
    d = torch.zeros_like(p)
    dense = torch.zeros_like(p)  # the gradient arriving at each expert's weight
    chosen = torch.zeros_like(p)
    rows = torch.arange(c["T"], device="cuda")
    for j in range(c["k"]):
        on = s["idx"][:, j] >= 0
        e = s["idx"][on, j].long()
        dense[rows[on], e] += g[on, j]
        chosen[rows[on], e] += 1.0
    ds = dense * s["scale"]
    if c["renorm"]:
        total = (p * chosen).sum(1, keepdim=True) + TINY
        ds = ds / total - chosen * s["scale"] * (dense * p).sum(1, keepdim=True) / total ** 2
    if c["score"] == "sigmoid":
        d = ds * p * torch.sigmoid(-s["logits"].double())
    elif c["renorm"]:  # sum of ds p is scale (g . p) / total * TINY / total: of its difference 64 bits would leave nothing
        d = p * (ds - s["scale"] * (dense * p).sum(1, keepdim=True) / total * (TINY / total))
    else:
        d = p * (ds - (ds * p).sum(1, keepdim=True))
    return dict(dlogits=d if s["add"] is None else d + s["add"].double())


def _exact_combine(s):
    c = s["c"]
    T, k = c["T"], c["k"]
    out = torch.zeros(T, c["cols"], dtype=torch.float64, device="cuda") if s["residual"] is None else s["residual"].double()
    for j in range(k):
        w = torch.ones(T, dtype=torch.float64, device="cuda") if s["w"] is None else s["w"][:, j].double()
        out += w[:, None] * s["y"][s["pos"][j: T * k: k].long()].double()
    for x in range(c["S"]):
        out += s["y"][s["pos"][T * k + x * T: T * k + (x + 1) * T].long()].double()
    return dict(out=out)


def _exact_combine_grad(s):
    c, d = s["c"], s["dout"].double()
    T, k = c["T"], c["k"]
    dw, rows = torch.empty(T, k, dtype=torch.float64, device="cuda"), torch.empty(s["y"].shape, dtype=torch.float64, device="cuda")
    for j in range(k):
        at = s["pos"][j: T * k: k].long()
        dw[:, j] = (d * s["y"][at].double()).sum(1)
        rows[at] = d * s["w"][:, j:j + 1].double()
    for x in range(c["S"]):
        rows[s["pos"][T * k + x * T: T * k + (x + 1) * T].long()] = d
    out = dict(dweight=dw)
    if c["dy"]:
        out["dy"] = rows
    if c["q"]:
        out["q"], out["scale"] = _exact_quant(rows)
    return out


def _exact_swiglu_grad(s):
    c, x, d = s["c"], s["x"].double(), s["dact"].double()
    gate, up = x[:, : c["cols"]], x[:, c["cols"]:]
    sig = torch.sigmoid(gate)
    dx = torch.cat([d * up * (sig + gate * sig * torch.sigmoid(-gate)), d * gate * sig], 1)
    out = {}
    if c["dx"]:
        out["dx"] = dx
    if c["q"]:
        out["q"], out["scale"] = _exact_quant(dx)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    form = dict(norm=_exact_norm, norm_grad=_exact_norm_grad, route=_exact_route, route_grad=_exact_route_grad, combine=_exact_combine,
                combine_grad=_exact_combine_grad, swiglu_grad=_exact_swiglu_grad)
    return form[case["op"]](s)
