// The weighted sum of a token's expert rows, and its gradients.
//   out[t] = sum_j w_tj y[pos(t, j)] + sum_s y[pos(s, t)] + residual[t];
//   dy[pos(t, j)] = w_tj dout[t],  dw_tj = dout[t] . y[pos(t, j)].
// Memory bound: every row is read once and every output written once.  Going by tokens
// rather than by rows makes the sum one of registers in a fixed order, and lets the gradient
// read dout once for all the token's rows.
#include "fp8_dev.h"

namespace mira {

namespace {

constexpr uint32_t kMaxGrid = 1u << 21;  // workgroups of a launch: fewer than 2^32 threads

struct CombineParams {
  const void* y;
  const float* w;       // may be null
  const int32_t* pos;
  const void* residual; // may be null
  void* out;
  size_t ldy, ld_res, ld_out;
  int T, k, S, cols, y_rows;
};

// A pair of token t: its position, -1 if it has none, and its weight.
struct Pair {
  int pos;
  float w;
};
__device__ __forceinline__ Pair pair_of(const int32_t* pos, const float* w, int T, int k, int y_rows, int t, int j) {
  const size_t at = j < k ? (size_t)t * k + j : (size_t)T * k + (size_t)(j - k) * T + t;
  const int p = pos[at];
  return Pair{(uint32_t)p < (uint32_t)y_rows ? p : -1, w && j < k ? w[at] : 1.f};
}

// A wave takes 512 columns of a token; a workgroup's four waves those of one token, or of
// two or four where rows are short (`share`: log2 of the waves that share a token).
template <typename Y, typename O>
__global__ __launch_bounds__(256) void combine_kernel(CombineParams p, int share) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int c = ((int)blockIdx.y * 4 + (wave & ((1 << share) - 1))) * 512 + lane * 8;
  const int step = gridDim.x * (4 >> share);
  for (int tw = blockIdx.x * (4 >> share) + (wave >> share); tw < p.T; tw += step) {
    const int t = __builtin_amdgcn_readfirstlane(tw);
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < p.k + p.S; ++j) {
      const Pair a = pair_of(p.pos, p.w, p.T, p.k, p.y_rows, t, j);
      if (a.pos < 0) continue;
      float v[8];
      load_cols((const Y*)p.y + (size_t)a.pos * p.ldy, c, p.cols, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] = fmaf(a.w, v[i], acc[i]);
    }
    if (p.residual) {
      float v[8];
      load_cols((const O*)p.residual + (size_t)t * p.ld_res, c, p.cols, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] += v[i];
    }
    store_cols((O*)p.out + (size_t)t * p.ld_out, c, p.cols, acc);
  }
}

struct CombineGradParams {
  const void* dout;
  const void* y;
  const float* w;  // may be null
  const int32_t* pos;
  void* dy;        // may be null
  uint8_t* q;      // may be null
  float* scale;
  float* dw;       // may be null
  size_t ld_dout, ldy, ld_dy, ldq, ld_s;
  int T, k, S, cols, y_rows;
  float q_eps;
};

// A workgroup takes a token, 2048 columns at a time; a wave's sums of products meet in LDS.
template <typename Y, typename O>
__global__ __launch_bounds__(256) void combine_grad_kernel(CombineGradParams p) {
  __shared__ float part[2][4][MIRA_MAX_TOPK];
  const int end = (int)align_up((size_t)p.cols, 2048);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int turn = 0;
  for (int t = blockIdx.x; t < p.T; t += gridDim.x, turn ^= 1) {
    float dot[MIRA_MAX_TOPK];
#pragma unroll
    for (int j = 0; j < MIRA_MAX_TOPK; ++j) dot[j] = 0.f;
    for (int c = threadIdx.x * 8; c < end; c += 2048) {
      float d[8];
      load_cols((const O*)p.dout + (size_t)t * p.ld_dout, c, p.cols, d);
      auto pair = [&](int j) {
        const Pair a = pair_of(p.pos, p.w, p.T, p.k, p.y_rows, t, j);
        float s = 0.f;
        if (a.pos < 0) return s;
        if (p.dw && j < p.k) {
          float v[8];
          load_cols((const Y*)p.y + (size_t)a.pos * p.ldy, c, p.cols, v);
#pragma unroll
          for (int i = 0; i < 8; ++i) s = fmaf(d[i], v[i], s);
        }
        if (p.dy || p.q) {
          float o[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] = a.w * d[i];
          if (p.dy) store_cols((Y*)p.dy + (size_t)a.pos * p.ld_dy, c, p.cols, o);
          if (p.q) quantize_block(o, c, p.cols, p.q_eps, p.q + (size_t)a.pos * p.ldq, p.scale + (size_t)a.pos * p.ld_s);
        }
        return s;
      };
#pragma unroll
      for (int j = 0; j < MIRA_MAX_TOPK; ++j)
        if (j < p.k) dot[j] += pair(j);
      for (int j = p.k; j < p.k + p.S; ++j) pair(j);
    }
    if (p.dw) {
#pragma unroll
      for (int j = 0; j < MIRA_MAX_TOPK; ++j)
        if (j < p.k) {
          const float s = lanes_reduce<64, AddOp>(dot[j]);
          if (lane == 0) part[turn][wave][j] = s;
        }
      __syncthreads();
      if ((int)threadIdx.x < p.k)
        p.dw[(size_t)t * p.k + threadIdx.x] = part[turn][0][threadIdx.x] + part[turn][1][threadIdx.x] + part[turn][2][threadIdx.x] +
                                              part[turn][3][threadIdx.x];
    }
  }
}

size_t or_dense(uint64_t ld, size_t dense) { return ld ? ld : dense; }

template <typename Y, typename O>
void launch_combine_of(const CombineParams& p, hipStream_t st) {
  const int parts = (p.cols + 511) / 512, share = parts == 1 ? 0 : parts == 2 ? 1 : 2;
  const uint32_t blocks = ((uint32_t)p.T + (4 >> share) - 1) / (4 >> share);
  launch_timed("combine", combine_kernel<Y, O>, dim3(blocks < kMaxGrid ? blocks : kMaxGrid, (parts + 3) / 4), dim3(256), 0, st, p, share);
}
template <typename Y, typename O>
void launch_combine_grad_of(const CombineGradParams& p, hipStream_t st) {
  launch_timed("combine_grad", combine_grad_kernel<Y, O>, dim3((uint32_t)p.T < kMaxGrid ? p.T : kMaxGrid), dim3(256), 0, st, p);
}

}  // namespace

hipError_t launch_combine(const mira_combine_args& a, hipStream_t st) {
  CombineParams p{};
  const size_t cols = a.cols;
  p.y = a.y;
  p.w = a.topk_weight;
  p.pos = a.pair_pos;
  p.residual = a.residual;
  p.out = a.out;
  p.ldy = or_dense(a.ldy, cols);
  p.ld_res = or_dense(a.ld_res, cols);
  p.ld_out = or_dense(a.ld_out, cols);
  p.T = a.n_tokens;
  p.k = a.top_k;
  p.S = a.n_shared;
  p.cols = a.cols;
  p.y_rows = a.y_rows;
  const bool yf = a.y_dtype == MIRA_F32, of = a.out_dtype == MIRA_F32;
  if (yf) of ? launch_combine_of<float, float>(p, st) : launch_combine_of<float, uint16_t>(p, st);
  else of ? launch_combine_of<uint16_t, float>(p, st) : launch_combine_of<uint16_t, uint16_t>(p, st);
  return hipGetLastError();
}

hipError_t launch_combine_grad(const mira_combine_grad_args& a, hipStream_t st) {
  CombineGradParams p{};
  const size_t cols = a.cols;
  p.dout = a.dout;
  p.y = a.y;
  p.w = a.topk_weight;
  p.pos = a.pair_pos;
  p.dy = a.dy;
  p.q = (uint8_t*)a.q;
  p.scale = a.scale;
  p.dw = a.dweight;
  p.ld_dout = or_dense(a.ld_dout, cols);
  p.ldy = or_dense(a.ldy, cols);
  p.ld_dy = or_dense(a.ld_dy, cols);
  p.ldq = or_dense(a.ldq, align_up(cols, 16));
  p.ld_s = or_dense(a.ld_scale, (cols + 127) / 128);
  p.T = a.n_tokens;
  p.k = a.top_k;
  p.S = a.n_shared;
  p.cols = a.cols;
  p.y_rows = a.y_rows;
  p.q_eps = a.q_eps;
  const bool yf = a.y_dtype == MIRA_F32, of = a.out_dtype == MIRA_F32;
  if (yf) of ? launch_combine_grad_of<float, float>(p, st) : launch_combine_grad_of<float, uint16_t>(p, st);
  else of ? launch_combine_grad_of<uint16_t, float>(p, st) : launch_combine_grad_of<uint16_t, uint16_t>(p, st);
  return hipGetLastError();
}

}  // namespace mira
