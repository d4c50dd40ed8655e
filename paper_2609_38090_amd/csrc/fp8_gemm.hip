// Product of e4m3 matrices with an fp32 scale per block of 128, one matrix or
// grouped over experts:
//   out[i][j] = sum_b xs[r][b] ws[j/128][b] * sum_{k in block b} x[r][k] w[j][k].
// The weight rows are the A operand and the token rows the B operand of 16 x 16
// tiles: a lane then holds four consecutive columns of one row of out, and its
// token scale is one value.
//
// The matrix cores' fp8 instructions do not sum in 32 bits: within each eight
// consecutive k, bits below 2^-13 of the largest product are dropped (measured
// on lone pairs of products; on normal data a block's sum is off by 1.3e-5 to
// 1.6e-5 of its 2-norm, 5e-5 with uniformly random bytes).  Products of e4m3
// values widened to bf16 (exact) sum to fp32 accuracy (1e-8).
#include "device_util.h"
#include "mira_internal.h"

namespace mira {

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

// Eight e4m3 bytes as bf16 (exact).
__device__ __forceinline__ v4i widen8(int lo, int hi) {
  v4i r;
  r[0] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false));
  r[1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true));
  r[2] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false));
  r[3] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true));
  return r;
}

// The 16 x 16 sums of one block, D = A(16 x 128) * B(128 x 16), through bf16.
// Lane l holds the same 32 k-values of A row l%16 and of B column l%16 (those
// of its k-group l/16); D row 4*(l/16)+i, column l%16.
__device__ __forceinline__ v4f block_bf16(v8i a, v8i b) {
  v4f d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < 4; ++s) d = mfma_bf16(widen8(a[2 * s], a[2 * s + 1]), widen8(b[2 * s], b[2 * s + 1]), d);
  return d;
}

struct GemmParams {
  const uint8_t* x;
  const float* xs;
  const uint8_t* w;
  const float* ws;
  const int32_t* offsets;
  const int32_t* order;
  void* out;
  size_t ldx, ld_xs, ldw, w_stride, ld_ws, ws_stride, ldo;
  int M, N, K, KB, G, x_rows, top_k;
};

struct Rows {
  int lo, hi;
};
__device__ __forceinline__ Rows rows_of(const GemmParams& p, int g) {
  if (!p.offsets) return Rows{0, p.M};
  const int lo = min(max(p.offsets[g], 0), p.M);
  return Rows{lo, min(max(p.offsets[g + 1], lo), p.M)};
}

// Source row of output row i; -1 for a row of zeros.
__device__ __forceinline__ int source_row(const GemmParams& p, int i) {
  if (!p.order) return i;
  const int pair = p.order[i];
  if (pair < 0) return -1;
  const int routed = p.x_rows * p.top_k;
  return pair < routed ? pair / p.top_k : (pair - routed) % p.x_rows;
}

__device__ __forceinline__ v8i join(v4i a, v4i b) {
  return v8i{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

// The 32 bytes from k on of a row (null: zeros); zeros from K on (a row's last
// 16 bytes are padded with zeros in memory).
__device__ __forceinline__ v8i load32(const uint8_t* row, int k, int K) {
  v4i a = zero16(), b = zero16();
  if (row && k < K) a = ld16(row + k);
  if (row && k + 16 < K) b = ld16(row + k + 16);
  return join(a, b);
}

template <typename OutT>
__device__ __forceinline__ void store_out(OutT* p, float v);
template <>
__device__ __forceinline__ void store_out<float>(float* p, float v) { *p = v; }
template <>
__device__ __forceinline__ void store_out<uint16_t>(uint16_t* p, float v) {
  *p = v != v ? (uint16_t)((__float_as_uint(v) >> 16) | 0x40u) : f32_to_bf16_rne(v);
}

// Few rows: a workgroup owns 16 weight rows of one group; its four waves split
// the blocks of the contraction and add up in LDS.
template <typename OutT>
__global__ __launch_bounds__(256) void fp8_gemm_rows_kernel(GemmParams p) {
  __shared__ float sums[4][16][17];
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63, r16 = lane & 15, kg = lane >> 4;
  const int g = blockIdx.y, n0 = blockIdx.x * 16;
  const Rows rows = rows_of(p, g);
  const int n = n0 + r16;
  const uint8_t* wrow = n < p.N ? p.w + g * p.w_stride + (size_t)n * p.ldw : nullptr;
  const float* wsc = p.ws + g * p.ws_stride + (size_t)(n0 >> 7) * p.ld_ws;
  OutT* out = (OutT*)p.out;
  const int per = (p.KB + 3) / 4, b0 = wave * per, b1 = min(b0 + per, p.KB);
  for (int m0 = rows.lo; m0 < rows.hi; m0 += 16) {
    const int m = m0 + r16;
    const int src = m < rows.hi ? source_row(p, m) : -1;
    const uint8_t* xrow = src >= 0 ? p.x + (size_t)src * p.ldx : nullptr;
    const float* xsc = src >= 0 ? p.xs + (size_t)src * p.ld_xs : nullptr;
    v4f acc = {0.f, 0.f, 0.f, 0.f};
    for (int b = b0; b < b1; ++b) {
      const v4f d = block_bf16(load32(wrow, b * 128 + kg * 32, p.K), load32(xrow, b * 128 + kg * 32, p.K));
      const float s = xsc ? xsc[b] * wsc[b] : 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = fmaf(d[i], s, acc[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[wave][r16][4 * kg + i] = acc[i];
    __syncthreads();
    const int mi = t >> 4, ni = t & 15;
    if (m0 + mi < rows.hi && n0 + ni < p.N)
      store_out(out + (size_t)(m0 + mi) * p.ldo + n0 + ni,
                (sums[0][mi][ni] + sums[1][mi][ni]) + (sums[2][mi][ni] + sums[3][mi][ni]));
    __syncthreads();
  }
}

}  // namespace

size_t fp8_gemm_ws_bytes(const mira_fp8_gemm_args& a) {
  (void)a;
  return 0;
}

hipError_t launch_fp8_gemm(const mira_fp8_gemm_args& a, hipStream_t st) {
  GemmParams p{};
  p.x = (const uint8_t*)a.x;
  p.xs = a.x_scale;
  p.w = (const uint8_t*)a.w;
  p.ws = a.w_scale;
  p.offsets = a.offsets;
  p.order = a.pair_order;
  p.out = a.out;
  p.M = a.m;
  p.N = a.n;
  p.K = a.k;
  p.KB = (a.k + 127) / 128;
  p.G = a.n_groups;
  p.x_rows = a.x_rows;
  p.top_k = a.top_k;
  const size_t k16 = align_up(a.k, 16), nb = ((size_t)a.n + 127) / 128;
  p.ldx = a.ldx ? a.ldx : k16;
  p.ldw = a.ldw ? a.ldw : k16;
  p.ld_xs = a.ld_xs ? a.ld_xs : p.KB;
  p.ld_ws = a.ld_ws ? a.ld_ws : p.KB;
  p.w_stride = a.w_stride ? a.w_stride : a.n * p.ldw;
  p.ws_stride = a.ws_stride ? a.ws_stride : nb * p.ld_ws;
  p.ldo = a.ldo ? a.ldo : a.n;
  const dim3 grid((p.N + 15) / 16, p.G);
  if (a.out_dtype == MIRA_F32)
    launch_timed("fp8_gemm_rows", fp8_gemm_rows_kernel<float>, grid, dim3(256), 0, st, p);
  else
    launch_timed("fp8_gemm_rows", fp8_gemm_rows_kernel<uint16_t>, grid, dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace mira
