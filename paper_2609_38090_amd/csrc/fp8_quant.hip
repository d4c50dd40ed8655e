// Quantizing to e4m3 with one fp32 scale per block of 1 x 128 or 128 x 128:
//   a = max(max |x|, eps), scale = fl32(a / 448), q = e4m3(fl32(x * fl32(448 / a))).
// Memory bound: every value is read once, kept in registers while its block's
// maximum is found, and written as one byte (a copy on this GPU runs at 5.1 TB/s:
// SwiGLU of 4096 x 2 x 14336 bf16, 296 MB, 56 us, 5.2 TB/s; 14336 x 4096 fp32 to both
// copies, 353 MB, 70 us, 5.1 TB/s; 8 x 4096, 5.4 us, is a launch).  A value is multiplied by the
// block's inverse instead of divided by its scale: one correctly rounded
// division per block instead of one per value (about ten instructions each).
#include "fp8_dev.h"

namespace mira {

namespace {

struct QuantParams {
  const void* x;
  uint8_t* q;
  uint8_t* qt;
  float* scale;
  float* scale_t;
  size_t ldx, ldq, ldqt, ld_s, ld_st;
  int rows, cols;
  float eps;
};

// silu(g) u.  exp(-g) = 2^t with the rounding of t = -g log2(e) carried in r (2
// steps), the quotient by the reciprocal instruction (1 step); a correctly rounded
// division and expf made this pass wait for them, 72 us for 4096 x 14336 bf16.
__device__ __forceinline__ float swiglu(float g, float u) {
  const float log2e = 1.44269502162933349609375f, rest = 1.92596299112661746887e-8f;
  const float t = -g * log2e;
  const float r = -fmaf(g, rest, fmaf(g, log2e, t));
  float e = __builtin_amdgcn_exp2f(t);
  // (above, e is infinite; below, it is nothing beside 1, and r infinite for gates whose t is)
  e = fabsf(t) < 128.f ? fmaf(e, r * 0.693147182464599609375f, e) : e;
  // (a quarter of 1 + e: the instruction gives 0 for a reciprocal below 2^-126, where g
  // times it is still a normal number)
  return g * (__builtin_amdgcn_rcpf(fmaf(e, 0.25f, 0.25f)) * 0.25f) * u;
}

// 1 x 128 blocks: 16 lanes hold a block, eight values each, so that a lane's load is
// 16 bytes of bf16 and its store 8, and the maximum is four exchanges of registers.
template <bool SWIGLU, typename T>
__global__ __launch_bounds__(256) void fp8_quant_rows_kernel(QuantParams p, int nb) {
  const size_t block = (size_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  const size_t total = (size_t)p.rows * nb;
  if (block >= total) return;  // whole groups of 16 lanes
  const size_t r = block / nb;
  const int b = (int)(block - r * nb), c = b * 128 + (threadIdx.x & 15) * 8;
  const T* row = (const T*)p.x + r * p.ldx;
  float v[8];
  load_cols(row, c, p.cols, v);
  if constexpr (SWIGLU) {
    float u[8];
    load_cols(row + p.cols, c, p.cols, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = swiglu(v[i], u[i]);
  }
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max_abs(m, v[i]);
  m = fmaxf(max16(m), p.eps);
  const float inv = kE4m3Max / m;
  if ((threadIdx.x & 15) == 0) p.scale[r * p.ld_s + b] = m / kE4m3Max;
  // the row's bytes reach up to the next multiple of 16
  if (c < (int)align_up((size_t)p.cols, 16)) {
    uint2 o;
    o.x = to_e4m3(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
    o.y = to_e4m3(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
    *(uint2*)(p.q + r * p.ldq + c) = o;
  }
}

// 128 x 128 blocks: a workgroup of 256 threads holds a block in registers,
// thread t columns 4 (t % 32) .. +3 of rows 4 (t / 32 + 8 j) .. +3, j < 4.  The
// transposed copy turns each 4 x 4 square of bytes with byte permutes and
// goes through LDS to rows of 16 bytes.
template <typename T>
__global__ __launch_bounds__(256) void fp8_quant_blocks_kernel(QuantParams p, int nb) {
  __shared__ float wave_m[4];
  __shared__ uint32_t turned[128][33];  // [column][row / 4], padded against bank conflicts
  const int t = threadIdx.x, cg = t & 31, rg = t >> 5;
  const int br = blockIdx.x / nb, bc = blockIdx.x - br * nb;
  const int c = bc * 128 + cg * 4;
  const T* x = (const T*)p.x;
  float v[4][4][4];
  float m = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = br * 128 + (rg + 8 * j) * 4 + i;
      load_cols(x + (size_t)min(r, p.rows - 1) * p.ldx, r < p.rows ? c : p.cols, p.cols, v[j][i]);
    }
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) m = max_abs(m, v[j][i][e]);
  m = wave_max(m);
  if ((t & 63) == 0) wave_m[t >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(fmaxf(wave_m[0], wave_m[1]), fmaxf(wave_m[2], wave_m[3])), p.eps);
  const float inv = kE4m3Max / m;
  if (t == 0) {
    p.scale[(size_t)br * p.ld_s + bc] = m / kE4m3Max;
    if (p.qt) p.scale_t[(size_t)bc * p.ld_st + br] = m / kE4m3Max;
  }
  const int cols16 = (int)align_up((size_t)p.cols, 16);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = br * 128 + (rg + 8 * j) * 4 + i;
      w[i] = to_e4m3(v[j][i][0] * inv, v[j][i][1] * inv, v[j][i][2] * inv, v[j][i][3] * inv);
      if (r < p.rows && c < cols16) *(uint32_t*)(p.q + (size_t)r * p.ldq + c) = w[i];
    }
    if (p.qt) {
      // bytes (w0.e, w1.e, w2.e, w3.e) of column e
      const uint32_t lo01 = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u);  // w0.0 w1.0 w0.1 w1.1
      const uint32_t hi01 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);  // w0.2 w1.2 w0.3 w1.3
      const uint32_t lo23 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);
      const uint32_t hi23 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
      turned[cg * 4 + 0][rg + 8 * j] = __builtin_amdgcn_perm(lo23, lo01, 0x05040100u);
      turned[cg * 4 + 1][rg + 8 * j] = __builtin_amdgcn_perm(lo23, lo01, 0x07060302u);
      turned[cg * 4 + 2][rg + 8 * j] = __builtin_amdgcn_perm(hi23, hi01, 0x05040100u);
      turned[cg * 4 + 3][rg + 8 * j] = __builtin_amdgcn_perm(hi23, hi01, 0x07060302u);
    }
  }
  if (!p.qt) return;
  __syncthreads();
  const int rows16 = (int)align_up((size_t)p.rows, 16);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int col = (t >> 3) + 32 * j, part = t & 7;
    if (bc * 128 + col < p.cols && br * 128 + part * 16 < rows16) {
      const uint32_t* s = &turned[col][part * 4];
      *(v4i*)(p.qt + (size_t)(bc * 128 + col) * p.ldqt + br * 128 + part * 16) =
          v4i{(int)s[0], (int)s[1], (int)s[2], (int)s[3]};
    }
  }
}

template <typename T>
void launch_quant(const mira_fp8_quant_args& a, const QuantParams& p, hipStream_t st) {
  const int nb = (p.cols + 127) / 128;
  if (a.block_rows == 128) {
    const dim3 grid((uint32_t)nb * ((p.rows + 127) / 128));
    launch_timed("fp8_quant_blocks", fp8_quant_blocks_kernel<T>, grid, dim3(256), 0, st, p, nb);
    return;
  }
  const dim3 grid((uint32_t)(((size_t)p.rows * nb + 15) / 16));
  if (a.flags & MIRA_FP8_SWIGLU)
    launch_timed("fp8_quant_rows", fp8_quant_rows_kernel<true, T>, grid, dim3(256), 0, st, p, nb);
  else
    launch_timed("fp8_quant_rows", fp8_quant_rows_kernel<false, T>, grid, dim3(256), 0, st, p, nb);
}

}  // namespace

hipError_t launch_fp8_quantize(const mira_fp8_quant_args& a, hipStream_t st) {
  const size_t nb = ((size_t)a.cols + 127) / 128, nr = ((size_t)a.rows + 127) / 128;
  QuantParams p{};
  p.x = a.x;
  p.q = (uint8_t*)a.q;
  p.qt = (uint8_t*)a.qt;
  p.scale = a.scale;
  p.scale_t = a.scale_t;
  p.ldx = a.ldx ? a.ldx : (size_t)a.cols * (a.flags & MIRA_FP8_SWIGLU ? 2 : 1);
  p.ldq = a.ldq ? a.ldq : align_up(a.cols, 16);
  p.ldqt = a.ldqt ? a.ldqt : align_up(a.rows, 16);
  p.ld_s = a.ld_scale ? a.ld_scale : nb;
  p.ld_st = a.ld_scale_t ? a.ld_scale_t : nr;
  p.rows = a.rows;
  p.cols = a.cols;
  p.eps = a.eps;
  if (a.x_dtype == MIRA_F32) launch_quant<float>(a, p, st);
  else launch_quant<uint16_t>(a, p, st);
  return hipGetLastError();
}

}  // namespace mira
