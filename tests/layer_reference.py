"""Plain 64-bit statements of the norm, the experts' selection, the combine and
SwiGLU's gradient, written from their formulas in numpy, for the tests; buffers
with guarded surroundings."""
import numpy as np
import torch

U32 = 2.0 ** -24           # half a step of fp32, relative
U16 = 2.0 ** -8            # of bf16
U8 = 2.0 ** -4             # of e4m3
TINY = 1e-20


def dt(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def unit(name):
    return U32 if name == "f32" else U16


def code(name):
    import paper_2609_38090_amd as mira
    return mira.MIRA_F32 if name == "f32" else mira.MIRA_BF16


def f64(t):
    return t.double().cpu().numpy()


class Guarded:
    """A matrix [rows][cols] with `ld` elements between rows, inside a buffer of a given byte
    that nothing may change outside of it.  `shift` elements before it change its alignment."""

    def __init__(self, rows, cols, dtype, ld=None, shift=0, fill=0xA5):
        self.rows, self.cols, self.ld, self.fill = rows, cols, ld or cols, fill
        es = torch.empty(0, dtype=dtype).element_size()
        self.at = 1024 // es + shift
        self.buf = torch.full((2048 + (shift + rows * self.ld) * es,), fill, dtype=torch.uint8, device="cuda")
        self.t = self.buf[:self.buf.numel() // es * es].view(dtype)[self.at:self.at + rows * self.ld].view(rows, self.ld)
        self.es = es

    def put(self, x):
        self.t[:, :self.cols] = x
        return self

    @property
    def v(self):
        return self.t[:, :self.cols]

    def intact(self, live=None):
        """Whether every byte outside the matrix's rows (of `live` columns) is as it was."""
        keep = torch.ones(self.buf.numel(), dtype=torch.bool, device="cuda")
        inner = keep[self.at * self.es:(self.at + self.rows * self.ld) * self.es].view(self.rows, self.ld * self.es)
        inner[:, :(live or self.cols) * self.es] = False
        return bool((self.buf[keep] == self.fill).all())


# ---- norm ------------------------------------------------------------------------

def norm(h, w, eps):
    """y and r of fp64 rows."""
    r = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    return h * r * w, r


def norm_grad(dy, dsum, h, w, eps):
    """dx, dweight and the magnitudes of their terms."""
    r = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    n, g = h * r, dy * w
    m = (n * g).mean(1, keepdims=True)
    dx = r * (g - n * m) + (0.0 if dsum is None else dsum)
    terms = r * (np.abs(g) + np.abs(n) * np.abs(n * g).mean(1, keepdims=True)) + (0.0 if dsum is None else np.abs(dsum))
    return dx, (dy * n).sum(0), terms, np.abs(dy * n).sum(0)


# ---- selection -----------------------------------------------------------------

def scores(x, sigmoid):
    with np.errstate(all="ignore"):
        if sigmoid:
            return np.where(x >= 0, 1.0 / (1.0 + np.exp(-np.abs(x))), np.exp(-np.abs(x)) / (1.0 + np.exp(-np.abs(x))))
        m = x.max(1, keepdims=True) if x.shape[1] else x
        e = np.exp(x - np.where(np.isneginf(m), 0.0, m))
        s = e.sum(1, keepdims=True)
        return np.where(s == 0, 0.0, e / np.where(s == 0, 1.0, s))


def select(x, k, sigmoid=False, renorm=False, bias=None, mask=None, groups=1, top_groups=1, best=1, scale=1.0):
    """idx [T][k] and weight [T][k] of fp64 logits, one comparison at a time."""
    T, E = x.shape
    s = scores(x, sigmoid)
    size = E // groups
    idx, weight = np.full((T, k), -1, np.int64), np.zeros((T, k))
    for t in range(T):
        if mask is not None and not mask[t]:
            continue
        can = [e for e in range(E) if not np.isnan(x[t, e]) and x[t, e] > -np.inf]
        c = {e: s[t, e] + bias[e] if bias is not None else x[t, e] for e in can}
        cg = {e: s[t, e] + bias[e] if bias is not None else s[t, e] if best == 2 else x[t, e] for e in can}
        if groups > 1:
            of = []
            for g in range(groups):
                mine = sorted((cg[e] for e in can if e // size == g), reverse=True)
                of.append(sum(mine[:best]) if mine else -np.inf)
            kept = sorted(range(groups), key=lambda g: (-of[g], g))[:top_groups]
            can = [e for e in can if e // size in kept]
        got = sorted(can, key=lambda e: (-c[e], e))[:k]
        idx[t, :len(got)] = got
        w = s[t, got]
        weight[t, :len(got)] = w * scale / (w.sum() + TINY) if renorm else w * scale
    return idx, weight


def pairs(idx, mask, E, S):
    """counts, offsets, order and positions of the pairs of idx and the shared experts."""
    T, k = idx.shape
    lists = [[] for _ in range(E + S)]
    for p, e in enumerate(idx.reshape(-1)):
        if e >= 0:
            lists[e].append(p)
    for s in range(S):
        lists[E + s] = [T * k + s * T + t for t in range(T) if mask is None or mask[t]]
    counts = np.array([len(v) for v in lists], np.int64)
    offsets = np.concatenate([[0], counts.cumsum()])
    flat = np.array([p for v in lists for p in v], np.int64)
    order, pos = np.full(T * (k + S), -1, np.int64), np.full(T * (k + S), -1, np.int64)
    order[:len(flat)] = flat
    pos[flat] = np.arange(len(flat))
    return counts, offsets, order, pos


def select_grad(x, idx, g, sigmoid, renorm, scale):
    """dlogits and the magnitudes of its terms; entries outside 0..E-1 count for nothing."""
    T, E = x.shape
    s = scores(x, sigmoid)
    d, mag = np.zeros((T, E)), np.zeros((T, E))
    for t in range(T):
        sel = [(j, e) for j, e in enumerate(idx[t]) if 0 <= e < E]
        if not sel:
            continue
        ds, dm = np.zeros(E), np.zeros(E)
        total = sum(s[t, e] for _, e in sel) + TINY
        a = sum(g[t, j] * s[t, e] for j, e in sel) / total
        am = sum(abs(g[t, j]) * s[t, e] for j, e in sel) / total
        for j, e in sel:
            ds[e] += scale * (g[t, j] - a) / total if renorm else scale * g[t, j]
            dm[e] += abs(scale) * (abs(g[t, j]) + am) / total if renorm else abs(scale * g[t, j])
        if sigmoid:
            d[t], mag[t] = ds * s[t] * (1.0 - s[t]), dm * s[t] * (1.0 - s[t])
        else:
            rest = scale * a * (TINY / total) if renorm else scale * sum(g[t, j] * s[t, e] for j, e in sel)
            restm = abs(scale) * (am * (TINY / total) if renorm else sum(abs(g[t, j]) * s[t, e] for j, e in sel))
            d[t], mag[t] = s[t] * (ds - rest), s[t] * (dm + restm)
    return d, mag


# ---- SwiGLU ----------------------------------------------------------------------

def swiglu_grad(gate, up, d):
    """dgate, dup and the magnitude of dgate's terms."""
    s, r = scores(gate, True), scores(-gate, True)
    return d * up * s * (1.0 + gate * r), d * gate * s, np.abs(d * up) * s * (1.0 + np.abs(gate * r))


def e4m3_close(q, scale, want, table, extra):
    """Whether codes q [rows][cols] with scale [rows][ceil(cols/128)] hold `want`: half a step of
    e4m3 (2^-4 of the value, or 2^-10 of the scale for its smallest numbers); `extra`, what the
    value was off before; fp32 roundings of 448/a, the product with it, a/448 and here."""
    s = np.repeat(scale, 128, axis=1)[:, :want.shape[1]].astype(np.float64)
    return np.abs(table[q] * s - want) <= U8 * np.abs(want) + 2.0 ** -10 * s + 2 * extra + 16 * U32 * np.abs(want)
