"""CPU checks of the balance loss, FP8 quantizer and FP8 product entry points:
argument structures, workspace sizes, and that bad calls are refused before any
launch (the pointers here are never dereferenced)."""
import pytest

import paper_2609_38090_amd as mira

ARG, SHAPE, ALIGN, WORKSPACE, UNSUPPORTED = -1, -2, -3, -4, -6


def _refused(call, args, code):
    with pytest.raises(mira.MiraError) as ei:
        call(args, stream=1)
    assert ei.value.code == code, str(ei.value)
    assert mira.mira_last_error()


def _balance(**kw):
    ws = mira.mira_balance_workspace_bytes(10, 8, 2)
    base = dict(logits=0x1000, topk_idx=0x2000, offsets=0x3000, n_tokens=10, n_experts=8, top_k=2, n_groups=2,
                coef=0.5, loss=0x4000, workspace=0x10000, workspace_bytes=ws)
    return mira.BalanceArgs(**{**base, **kw})


@pytest.mark.parametrize("bad,code", [
    (dict(logits_dtype=5), ARG), (dict(n_experts=0), SHAPE), (dict(n_experts=257), SHAPE), (dict(top_k=0), SHAPE),
    (dict(top_k=17), SHAPE), (dict(n_tokens=-1), SHAPE), (dict(n_tokens=2 ** 30), SHAPE), (dict(n_groups=0), SHAPE),
    (dict(n_groups=2 ** 21 + 1), SHAPE), (dict(offsets=None), ARG), (dict(coef=float("nan")), ARG), (dict(coef=float("inf")), ARG),
    (dict(ld_logits=7), SHAPE), (dict(ld_dlogits=7), SHAPE), (dict(logits=None), ARG), (dict(topk_idx=None), ARG),
    (dict(logits=0x1002), ALIGN), (dict(loss=0x4001), ALIGN), (dict(workspace=None), ARG),
    (dict(workspace=0x10010), ALIGN), (dict(workspace_bytes=16), WORKSPACE),
    (dict(dlogits=0x1000, ld_logits=12, ld_dlogits=8), ARG), (dict(ld_logits=2 ** 40), SHAPE),
])
def test_balance_refuses(bad, code):
    _refused(mira.mira_balance_loss, _balance(**bad), code)


def test_balance_workspace():
    sizes = [mira.mira_balance_workspace_bytes(100, 64, g) for g in (1, 2, 100, 5000)]
    assert sizes == sorted(sizes) and all(s % 256 == 0 for s in sizes)
    for bad in ((-1, 8, 1), (4, 0, 1), (4, 257, 1), (4, 8, 0), (4, 8, 2 ** 21 + 1)):
        with pytest.raises(mira.MiraError):
            mira.mira_balance_workspace_bytes(*bad)


def _quant(**kw):
    base = dict(x=0x1000, rows=10, cols=200, q=0x2000, scale=0x3000)
    return mira.Fp8QuantArgs(**{**base, **kw})


@pytest.mark.parametrize("bad,code", [
    (dict(x_dtype=2), ARG), (dict(flags=2), ARG), (dict(block_rows=64), ARG), (dict(rows=-1), SHAPE),
    (dict(cols=0), SHAPE), (dict(eps=0.0), ARG), (dict(eps=float("nan")), ARG), (dict(eps=1e-38), ARG),
    (dict(ldx=199), SHAPE), (dict(flags=mira.MIRA_FP8_SWIGLU, ldx=399), SHAPE), (dict(ldq=200), SHAPE),
    (dict(ldq=216), ALIGN), (dict(ld_scale=1), SHAPE), (dict(x=None), ARG), (dict(q=None), ARG),
    (dict(scale=None), ARG), (dict(q=0x2008), ALIGN), (dict(x=0x1001), ALIGN), (dict(scale=0x3002), ALIGN),
    (dict(qt=0x5000, scale_t=0x6000), UNSUPPORTED), (dict(block_rows=128, qt=0x5000), ARG),
    (dict(block_rows=128, scale_t=0x5000), ARG), (dict(block_rows=128, flags=mira.MIRA_FP8_SWIGLU), UNSUPPORTED),
    (dict(block_rows=128, qt=0x5000, scale_t=0x6000, ldqt=8), SHAPE),
    (dict(block_rows=128, qt=0x5008, scale_t=0x6000), ALIGN), (dict(rows=2 ** 30, cols=2 ** 20), SHAPE),
])
def test_quantize_refuses(bad, code):
    _refused(mira.mira_fp8_quantize, _quant(**bad), code)


def _gemm(**kw):
    base = dict(m=10, n=200, k=300, x=0x1000, x_scale=0x2000, x_rows=10, w=0x3000, w_scale=0x4000, out=0x5000,
                workspace=0x100000, workspace_bytes=2 ** 40)
    return mira.Fp8GemmArgs(**{**base, **kw})


@pytest.mark.parametrize("bad,code", [
    (dict(m=-1), SHAPE), (dict(n=0), SHAPE), (dict(k=0), SHAPE), (dict(n_groups=0), SHAPE),
    (dict(n_groups=257, offsets=0x9000), SHAPE), (dict(n_groups=2), ARG), (dict(out_dtype=9), ARG),
    (dict(x_rows=9), SHAPE), (dict(top_k=1), ARG), (dict(pair_order=0x6000), SHAPE),
    (dict(pair_order=0x6000, top_k=17), SHAPE), (dict(pair_order=0x6000, top_k=2, x_rows=0), SHAPE),
    (dict(ldx=300), SHAPE), (dict(ldx=312), ALIGN), (dict(ldw=296), SHAPE), (dict(ld_xs=2), SHAPE),
    (dict(ld_ws=2), SHAPE), (dict(ldo=199), SHAPE), (dict(w_stride=1600), SHAPE), (dict(w_stride=60808), ALIGN),
    (dict(ws_stride=5), SHAPE), (dict(x=None), ARG), (dict(x_scale=None), ARG), (dict(w=None), ARG),
    (dict(w_scale=None), ARG), (dict(out=None), ARG), (dict(x=0x1008), ALIGN), (dict(w=0x3004), ALIGN),
    (dict(out=0x5001), ALIGN), (dict(x_scale=0x2002), ALIGN),
])
def test_gemm_refuses(bad, code):
    _refused(mira.mira_fp8_gemm, _gemm(**bad), code)


def test_gemm_workspace():
    assert mira.mira_fp8_gemm_workspace_bytes(_gemm(m=0)) == 0
    for bad in (dict(m=-1), dict(n=0), dict(k=0), dict(n_groups=2)):
        with pytest.raises(mira.MiraError):
            mira.mira_fp8_gemm_workspace_bytes(_gemm(**bad))
    big = _gemm(m=8, n=64, k=8192)
    need = mira.mira_fp8_gemm_workspace_bytes(big)
    if need:  # a call that splits its contraction refuses a smaller or misaligned workspace
        for bad, code in ((dict(workspace_bytes=need - 1), WORKSPACE), (dict(workspace=0x100010), ALIGN),
                          (dict(workspace=None), ARG)):
            _refused(mira.mira_fp8_gemm, _gemm(m=8, n=64, k=8192, x_rows=8, **bad), code)


def test_empty_calls_are_no_ops():
    mira.mira_fp8_quantize(_quant(rows=0, x=None, q=None, scale=None), stream=1)
    mira.mira_fp8_gemm(_gemm(m=0, x=None, w=None, out=None), stream=1)


def test_gemm_workspace_refusals():
    """A call that splits its contraction refuses a smaller, misaligned or missing workspace,
    with groups and without."""
    for kw in (dict(m=20, n=260, k=9000, x_rows=20), dict(m=97, n=130, k=9000, x_rows=97, n_groups=4, offsets=0x9000)):
        for dt in (mira.MIRA_F32, mira.MIRA_BF16):
            need = mira.mira_fp8_gemm_workspace_bytes(_gemm(out_dtype=dt, **kw))
            assert need > 0 and need % (4 * kw["m"] * kw["n"]) == 0
            for bad, code in ((dict(workspace_bytes=need - 1), WORKSPACE), (dict(workspace_bytes=0), WORKSPACE),
                              (dict(workspace=0x100010), ALIGN), (dict(workspace=None), ARG)):
                _refused(mira.mira_fp8_gemm, _gemm(out_dtype=dt, **kw, **bad), code)
