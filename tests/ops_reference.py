"""Plain 64-bit statements of the balance loss, the FP8 quantizer and the FP8
product, written from their formulas in numpy and torch, for the tests."""
import numpy as np
import torch

U32 = 2.0 ** -24  # half a step of fp32, relative
U16 = 2.0 ** -8   # of bf16


def e4m3_table():
    """The value of each of the 256 e4m3 codes (0x7f and 0xff are NaN)."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e.astype(np.float64) - 10))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


TABLE = e4m3_table()
_POS = TABLE[:127]  # ascending, codes 0..126


def e4m3_codes(v):
    """Codes of the e4m3 values nearest to v (64-bit), ties to the even code."""
    v = np.asarray(v, np.float64)
    a = np.abs(v)
    hi = np.clip(np.searchsorted(_POS, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _POS[lo], _POS[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(a >= 448.0, 126, code)
    code = np.where(np.isnan(v), 127, code)
    return (code | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def quantize(x, block_rows, eps):
    """(codes [rows][cols], scales) of an fp32 array, by the definition: fp32
    divisions and product, nearest e4m3."""
    x = np.asarray(x, np.float32)
    rows, cols = x.shape
    nr, nc = -(-rows // block_rows), -(-cols // 128)
    full = np.zeros((nr * block_rows, nc * 128), np.float32)
    full[:rows, :cols] = x
    v = full.reshape(nr, block_rows, nc, 128)
    a = np.maximum(np.nanmax(np.abs(v), axis=(1, 3)), np.float32(eps)).astype(np.float32)
    top = np.float32(448)
    with np.errstate(invalid="ignore"):
        q = e4m3_codes((v * (top / a)[:, None, :, None]).astype(np.float32))
    return q.reshape(nr * block_rows, nc * 128)[:rows, :cols], a / top


def balance(logits, idx, offsets, mask, coef, grad_loss):
    """loss, counts, mean_prob, dlogits (fp64 numpy) of fp64 logits [T][E]."""
    T, E = logits.shape
    k, G = idx.shape[1], len(offsets) - 1
    with np.errstate(all="ignore"):
        m = logits.max(1, keepdims=True) if E else logits
        m = np.where(np.isneginf(m), 0.0, m)
        e = np.exp(logits - m)
        s = e.sum(1, keepdims=True)
        p = np.where(s == 0, 0.0, e / np.where(s == 0, 1.0, s))
    loss, counts, mean, d = np.zeros(G), np.zeros((G, E), np.int64), np.zeros((G, E)), np.full((T, E), np.nan)
    for g in range(G):
        rows = np.arange(offsets[g], offsets[g + 1])
        kept = rows[mask[rows] != 0] if len(rows) else rows
        d[rows] = 0.0
        n = len(kept)
        if not n:
            continue
        sel = idx[kept].reshape(-1)
        counts[g] = np.bincount(sel[(sel >= 0) & (sel < E)], minlength=E)
        mean[g] = p[kept].mean(0)
        f = counts[g] * E / (k * n)
        loss[g] = coef * (f * mean[g]).sum()
        d[kept] = grad_loss[g] * coef / n * p[kept] * (f - (p[kept] * f).sum(1, keepdims=True))
    return loss, counts, mean, d


def dequantize(codes, scale, block_rows, rows, cols):
    """fp64 torch values of codes [rows][>=cols] (uint8) with their scales, and the same with magnitudes."""
    t = torch.from_numpy(TABLE).to(codes.device)
    s = scale.double().repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :cols]
    return t[codes[:rows, :cols].long()] * s


def source_rows(order, x_rows, top_k):
    p = order.long()
    r = torch.where(p < x_rows * top_k, torch.div(p, top_k, rounding_mode="floor"), (p - x_rows * top_k) % x_rows)
    return torch.where(p < 0, -torch.ones_like(p), r)


def gemm(x, w):
    """x w^T and |x| |w|^T in fp64 on the CPU."""
    x, w = x.cpu(), w.cpu()
    return x @ w.t(), x.abs() @ w.abs().t()


def gemm_bound(mag, k, bf16, value):
    """Largest error of the product's sums: a block's 128 products and its two
    scales in fp32, the blocks' sums, one rounding of the output.

    With bf16 output the sums inside a block may come from the fp8 matrix
    instructions, which add each eight consecutive products after dropping, toward
    zero, the bits below 2^(E-13), E the sum of the exponents of the largest of
    them.  That quantum is at most 2^-13 of the largest product, eight products
    lose less than one quantum each, so eight products' sum is off by less than
    8 * 2^-13 = 2^-10 of the largest product, hence of their magnitudes' sum; the
    same factor holds for the scaled sum over all of them."""
    kb = -(-k // 128)
    sums = (128 + kb + 8) * U32 * mag * (1 + 2 * U16)
    return sums + ((U16 * (value.abs() + 2.0 ** -10 * mag) + 2.0 ** -10 * mag) if bf16 else U32 * value.abs()) + 1e-37
