// Host entry points of the operators around the expert step (balance loss,
// FP8 quantizing and product): argument checks and dispatch.  Every check runs
// before any launch.
#include <cmath>
#include <cstdint>

#include "mira.h"
#include "mira_internal.h"

namespace {

using mira::clear_error;
using mira::set_error;

bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
bool known_dtype(int32_t d) { return d == MIRA_F32 || d == MIRA_BF16; }
size_t esize(int32_t d) { return d == MIRA_F32 ? 4 : 2; }
uint64_t blocks(uint64_t n) { return (n + MIRA_FP8_BLOCK - 1) / MIRA_FP8_BLOCK; }
uint64_t pad16(uint64_t n) { return (n + 15) / 16 * 16; }

// Strides may not take any buffer past 2^60 bytes, so that no offset overflows.
constexpr uint64_t kMaxLd = 1ull << 28;

// Groups of a balance loss: a workgroup of 1024 threads each, fewer than 2^32 in a launch.
constexpr int32_t kMaxGroups = 1 << 21;

int check_ld(const char* name, uint64_t ld, uint64_t least, uint64_t mult) {
  if (ld == 0) return MIRA_OK;
  if (ld < least)
    return set_error(MIRA_ERR_SHAPE, "%s (%llu) must be at least %llu", name, (unsigned long long)ld,
                     (unsigned long long)least);
  if (ld > kMaxLd) return set_error(MIRA_ERR_SHAPE, "%s (%llu) is too large", name, (unsigned long long)ld);
  if (ld % mult)
    return set_error(MIRA_ERR_ALIGN, "%s (%llu) must be a multiple of %llu", name, (unsigned long long)ld,
                     (unsigned long long)mult);
  return MIRA_OK;
}

int hip_result(hipError_t e, const char* what) {
  if (e != hipSuccess) return set_error(MIRA_ERR_HIP, "%s failed: %s", what, hipGetErrorString(e));
  return clear_error();
}

int check_gemm_sizes(const mira_fp8_gemm_args* a) {
  if (!a) return set_error(MIRA_ERR_ARG, "args is NULL");
  if (a->reserved != 0) return set_error(MIRA_ERR_ARG, "reserved must be 0");
  if (!known_dtype(a->out_dtype)) return set_error(MIRA_ERR_ARG, "out_dtype must be MIRA_F32 or MIRA_BF16");
  if (a->m < 0 || a->m > 1 << 28) return set_error(MIRA_ERR_SHAPE, "m (%d) must be in [0, 2^28]", a->m);
  if (a->n < 1 || a->n > 1 << 24) return set_error(MIRA_ERR_SHAPE, "n (%d) must be in [1, 2^24]", a->n);
  if (a->k < 1 || a->k > 1 << 24) return set_error(MIRA_ERR_SHAPE, "k (%d) must be in [1, 2^24]", a->k);
  if (a->n_groups < 1 || a->n_groups > MIRA_MAX_EXPERTS)
    return set_error(MIRA_ERR_SHAPE, "n_groups (%d) must be in [1, %d]", a->n_groups, MIRA_MAX_EXPERTS);
  if (!a->offsets && a->n_groups != 1) return set_error(MIRA_ERR_ARG, "several groups need offsets");
  if (a->m > 0 && !mira::fp8_gemm_fits(*a))
    return set_error(MIRA_ERR_SHAPE, "m, n and n_groups (%d, %d, %d) are too large together", a->m, a->n, a->n_groups);
  return MIRA_OK;
}

}  // namespace

extern "C" {

size_t mira_balance_workspace_bytes(int32_t max_tokens, int32_t n_experts, int32_t max_groups) {
  if (max_tokens < 0 || n_experts < 1 || n_experts > MIRA_MAX_EXPERTS || max_groups < 1 || max_groups > kMaxGroups) return 0;
  return mira::balance_ws_bytes(n_experts, max_groups);
}

int mira_balance_loss(const mira_balance_args* a, hipStream_t stream) {
  if (!a) return set_error(MIRA_ERR_ARG, "args is NULL");
  if (!known_dtype(a->logits_dtype)) return set_error(MIRA_ERR_ARG, "logits_dtype must be MIRA_F32 or MIRA_BF16");
  if (a->n_experts < 1 || a->n_experts > MIRA_MAX_EXPERTS)
    return set_error(MIRA_ERR_SHAPE, "n_experts (%d) must be in [1, %d]", a->n_experts, MIRA_MAX_EXPERTS);
  if (a->top_k < 1 || a->top_k > MIRA_MAX_TOPK)
    return set_error(MIRA_ERR_SHAPE, "top_k (%d) must be in [1, %d]", a->top_k, MIRA_MAX_TOPK);
  if (a->n_tokens < 0 || (int64_t)a->n_tokens * a->top_k > (int64_t)1 << 30)
    return set_error(MIRA_ERR_SHAPE, "n_tokens (%d) must be in [0, 2^30 / top_k]", a->n_tokens);
  if (a->n_groups < 1 || a->n_groups > kMaxGroups)
    return set_error(MIRA_ERR_SHAPE, "n_groups (%d) must be in [1, 2^21]", a->n_groups);
  if (!a->offsets && a->n_groups != 1) return set_error(MIRA_ERR_ARG, "several groups need offsets");
  if (!std::isfinite(a->coef)) return set_error(MIRA_ERR_ARG, "coef must be finite");
  int rc = check_ld("ld_logits", a->ld_logits, a->n_experts, 1);
  if (!rc) rc = check_ld("ld_dlogits", a->ld_dlogits, a->n_experts, 1);
  if (rc) return rc;
  if (a->n_tokens > 0 && (!a->logits || !a->topk_idx))
    return set_error(MIRA_ERR_ARG, "logits and topk_idx are required");
  const size_t esz = esize(a->logits_dtype);
  if (!aligned(a->logits, esz) || !aligned(a->dlogits, esz) || !aligned(a->topk_idx, 4) ||
      !aligned(a->offsets, 4) || !aligned(a->grad_loss, 4) || !aligned(a->counts, 4) ||
      !aligned(a->mean_prob, 4) || !aligned(a->loss, 4))
    return set_error(MIRA_ERR_ALIGN, "a pointer is not aligned to its element type");
  if (a->dlogits && a->dlogits == a->logits) {
    const uint64_t E = a->n_experts;
    if ((a->ld_logits ? a->ld_logits : E) != (a->ld_dlogits ? a->ld_dlogits : E))
      return set_error(MIRA_ERR_ARG, "dlogits over logits needs equal row strides");
  }
  if (!a->workspace) return set_error(MIRA_ERR_ARG, "workspace is NULL");
  if (!aligned(a->workspace, 256)) return set_error(MIRA_ERR_ALIGN, "workspace must be 256-byte aligned");
  const size_t need = mira::balance_ws_bytes(a->n_experts, a->n_groups);
  if (a->workspace_bytes < need)
    return set_error(MIRA_ERR_WORKSPACE, "workspace has %llu bytes, %zu needed",
                     (unsigned long long)a->workspace_bytes, need);
  return hip_result(mira::launch_balance(*a, stream), "balance loss launch");
}

int mira_fp8_quantize(const mira_fp8_quant_args* a, hipStream_t stream) {
  if (!a) return set_error(MIRA_ERR_ARG, "args is NULL");
  if (!known_dtype(a->x_dtype)) return set_error(MIRA_ERR_ARG, "x_dtype must be MIRA_F32 or MIRA_BF16");
  if (a->flags & ~MIRA_FP8_SWIGLU) return set_error(MIRA_ERR_ARG, "unknown flag bits 0x%x", a->flags & ~MIRA_FP8_SWIGLU);
  if (a->block_rows != 1 && a->block_rows != MIRA_FP8_BLOCK)
    return set_error(MIRA_ERR_ARG, "block_rows (%d) must be 1 or %d", a->block_rows, MIRA_FP8_BLOCK);
  const bool swiglu = a->flags & MIRA_FP8_SWIGLU, weights = a->block_rows != 1;
  if (swiglu && weights) return set_error(MIRA_ERR_UNSUPPORTED, "MIRA_FP8_SWIGLU quantizes rows (block_rows 1)");
  if (a->rows < 0) return set_error(MIRA_ERR_SHAPE, "rows must be >= 0");
  if (a->cols < 1 || a->cols > 1 << 24) return set_error(MIRA_ERR_SHAPE, "cols (%d) must be in [1, 2^24]", a->cols);
  if (!(a->eps >= 1e-30f && a->eps <= 1e30f)) return set_error(MIRA_ERR_ARG, "eps must be in [1e-30, 1e30]");
  const uint64_t nb = blocks(a->cols), nr = blocks(a->rows);
  // threads of one launch stay below 2^32
  if ((weights ? nr * nb > 1ull << 23 : (uint64_t)a->rows * nb > 1ull << 27))
    return set_error(MIRA_ERR_SHAPE, "too many blocks (%d rows, %d columns)", a->rows, a->cols);
  if (!!a->qt != !!a->scale_t) return set_error(MIRA_ERR_ARG, "qt and scale_t go together");
  if (a->qt && !weights) return set_error(MIRA_ERR_UNSUPPORTED, "the transposed copy needs block_rows 128");
  int rc = check_ld("ldx", a->ldx, (uint64_t)a->cols * (swiglu ? 2 : 1), 1);
  if (!rc) rc = check_ld("ldq", a->ldq, pad16(a->cols), 16);
  if (!rc) rc = check_ld("ld_scale", a->ld_scale, nb, 1);
  if (!rc) rc = check_ld("ldqt", a->ldqt, pad16(a->rows), 16);
  if (!rc) rc = check_ld("ld_scale_t", a->ld_scale_t, nr, 1);
  if (rc) return rc;
  if (a->rows == 0) return clear_error();
  if (!a->x || !a->q || !a->scale) return set_error(MIRA_ERR_ARG, "x, q and scale are required");
  if (!aligned(a->q, 16) || !aligned(a->qt, 16)) return set_error(MIRA_ERR_ALIGN, "q and qt must be 16-byte aligned");
  if (!aligned(a->x, esize(a->x_dtype)) || !aligned(a->scale, 4) || !aligned(a->scale_t, 4))
    return set_error(MIRA_ERR_ALIGN, "a pointer is not aligned to its element type");
  return hip_result(mira::launch_fp8_quantize(*a, stream), "fp8 quantize launch");
}

size_t mira_fp8_gemm_workspace_bytes(const mira_fp8_gemm_args* a) {
  if (check_gemm_sizes(a)) return SIZE_MAX;
  clear_error();
  return a->m == 0 ? 0 : mira::fp8_gemm_ws_bytes(*a);
}

int mira_fp8_gemm(const mira_fp8_gemm_args* a, hipStream_t stream) {
  int rc = check_gemm_sizes(a);
  if (rc) return rc;
  if (a->pair_order) {
    if (a->top_k < 1 || a->top_k > MIRA_MAX_TOPK)
      return set_error(MIRA_ERR_SHAPE, "top_k (%d) must be in [1, %d] with pair_order", a->top_k, MIRA_MAX_TOPK);
    if (a->x_rows < (a->m > 0 ? 1 : 0) || (int64_t)a->x_rows * a->top_k > (int64_t)1 << 30)
      return set_error(MIRA_ERR_SHAPE, "x_rows (%d) must be in [1, 2^30 / top_k]", a->x_rows);
  } else {
    if (a->top_k != 0) return set_error(MIRA_ERR_ARG, "top_k must be 0 without pair_order");
    if (a->x_rows < a->m) return set_error(MIRA_ERR_SHAPE, "x_rows (%d) must be at least m (%d)", a->x_rows, a->m);
  }
  const uint64_t k16 = pad16(a->k), kb = blocks(a->k), nb = blocks(a->n);
  rc = check_ld("ldx", a->ldx, k16, 16);
  if (!rc) rc = check_ld("ldw", a->ldw, k16, 16);
  if (!rc) rc = check_ld("ld_xs", a->ld_xs, kb, 1);
  if (!rc) rc = check_ld("ld_ws", a->ld_ws, kb, 1);
  if (!rc) rc = check_ld("ldo", a->ldo, a->n, 1);
  if (rc) return rc;
  if (a->ldx > 1 << 24 || a->ldw > 1 << 24) return set_error(MIRA_ERR_SHAPE, "ldx and ldw must be at most 2^24");
  const uint64_t ldw = a->ldw ? a->ldw : k16, ld_ws = a->ld_ws ? a->ld_ws : kb;
  if (a->w_stride && (a->w_stride < (a->n - 1) * ldw + k16 || a->w_stride > 1ull << 50))
    return set_error(MIRA_ERR_SHAPE, "w_stride (%llu) is smaller than a matrix, or too large", (unsigned long long)a->w_stride);
  if (a->w_stride % 16) return set_error(MIRA_ERR_ALIGN, "w_stride must be a multiple of 16");
  if (a->ws_stride && (a->ws_stride < (nb - 1) * ld_ws + kb || a->ws_stride > 1ull << 48))
    return set_error(MIRA_ERR_SHAPE, "ws_stride (%llu) is smaller than a matrix's scales, or too large", (unsigned long long)a->ws_stride);
  if (a->m == 0) return clear_error();
  if (!a->x || !a->x_scale || !a->w || !a->w_scale || !a->out)
    return set_error(MIRA_ERR_ARG, "x, x_scale, w, w_scale and out are required");
  if (!aligned(a->x, 16) || !aligned(a->w, 16)) return set_error(MIRA_ERR_ALIGN, "x and w must be 16-byte aligned");
  if (!aligned(a->x_scale, 4) || !aligned(a->w_scale, 4) || !aligned(a->offsets, 4) ||
      !aligned(a->pair_order, 4) || !aligned(a->out, esize(a->out_dtype)))
    return set_error(MIRA_ERR_ALIGN, "a pointer is not aligned to its element type");
  const size_t need = mira::fp8_gemm_ws_bytes(*a);
  if (need && !a->workspace) return set_error(MIRA_ERR_ARG, "workspace is NULL, %zu bytes needed", need);
  if (need && !aligned(a->workspace, 256)) return set_error(MIRA_ERR_ALIGN, "workspace must be 256-byte aligned");
  if (a->workspace_bytes < need)
    return set_error(MIRA_ERR_WORKSPACE, "workspace has %llu bytes, %zu needed",
                     (unsigned long long)a->workspace_bytes, need);
  return hip_result(mira::launch_fp8_gemm(*a, stream), "fp8 product launch");
}

}  // extern "C"
