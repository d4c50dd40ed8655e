// The weighted sum of a token's expert rows, and its gradients.
//   out[t] = sum_j w_tj y[pos(t, j)] + sum_s y[pos(s, t)] + residual[t];
//   dy[pos(t, j)] = w_tj dout[t],  dw_tj = dout[t] . y[pos(t, j)].
// Memory bound: every row is read once and every output written once.  Going by tokens
// rather than by rows makes the sum one of registers in a fixed order, and lets the gradient
// read dout once for all the token's rows.  4096 tokens of 2 x 4096 bf16 with a residual 27.5 us (134 MB,
// 4.9 TB/s; a copy of 1 GB reaches 5.2); the gradient of 2048 tokens of 8 x 2048 bf16, to e4m3 and the
// weights, 21.8 us (93 MB, 4.3 TB/s).
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

// The pairs of a token, one to a lane (further ones as they are asked for); j is the same for the
// whole wave.
struct TokenPairs {
  const int32_t* pos;
  const float* w;
  int T, k, y_rows, t;
  Pair held{-1, 0.f};
  __device__ __forceinline__ TokenPairs(const int32_t* pos, const float* w, int T, int k, int S, int y_rows, int t)
      : pos(pos), w(w), T(T), k(k), y_rows(y_rows), t(t) {
    const int lane = threadIdx.x & 63;
    if (lane < k + S) held = pair_of(pos, w, T, k, y_rows, t, lane);
  }
  __device__ __forceinline__ Pair operator[](int j) const {
    if (j >= 64) return pair_of(pos, w, T, k, y_rows, t, j);
    return Pair{__builtin_amdgcn_readlane(held.pos, j), __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(held.w), j))};
  }
};

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
    const TokenPairs all(p.pos, p.w, p.T, p.k, p.S, p.y_rows, t);
    Raw8<O> res;
    if (p.residual) load_raw((const O*)p.residual + (size_t)t * p.ld_res, c, p.cols, res);
    for (int j0 = 0; j0 < p.k + p.S; j0 += 4) {
      Raw8<Y> v[4];
      if (p.y_rows > 0) {
#pragma unroll
        for (int u = 0; u < 4; ++u)  // (a row of any pair beyond the last, or without a position)
          load_raw((const Y*)p.y + (size_t)max(all[min(j0 + u, p.k + p.S - 1)].pos, 0) * p.ldy, c, p.cols, v[u]);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (j0 + u >= p.k + p.S) continue;
        const Pair a = all[j0 + u];
        if (a.pos < 0) continue;
        settle(v[u], c, p.cols);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = fmaf(a.w, v[u][i], acc[i]);
      }
    }
    if (p.residual) {
      settle(res, c, p.cols);
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] += res[i];
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

// 2^share waves take a token, 512 columns each at a time; their sums of products meet in LDS.  A
// workgroup has four waves, or 16 for one token where tokens are few and rows long (9 pairs a token, us
// with four and 16 waves: 2 tokens of 14595 columns 33 and 18; 256 of 2304 12.4 and 9.5, of 14595 41 and
// 26; 400 of 2304 14.1 and 16.6, of 14595 54 and 47).  A token's positions and weights are loaded at
// once, one to a lane, and so are four pairs' rows (2048 tokens of 8 x 2048: 28 us with each pair's loads
// behind the last one's, 25 so, eight pairs' rows at once the same; 22 with rows' ends loaded without a
// branch).
// The blocks' maxima of w dout are w times those of dout, rounding being monotonic, so a block is
// searched once for all the token's pairs.
template <int K, typename Y, typename O>
__global__ __launch_bounds__(1024) void combine_grad_kernel(CombineGradParams p, int share) {
  constexpr int NB = 4;
  __shared__ float part[2][16][K];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, per = ((int)blockDim.x >> 6) >> share;  // tokens of a workgroup
  const int first = wave & ((1 << share) - 1), span = 512 << share;
  const int end = (int)align_up((size_t)p.cols, 512), pairs = p.k + p.S;
  const bool dots = p.dw && p.y_rows > 0;
  int turn = 0;
  for (int t0 = blockIdx.x * per; t0 < p.T; t0 += gridDim.x * per, turn ^= 1) {
    const int t = __builtin_amdgcn_readfirstlane(t0 + (wave >> share));
    float dot[K];
#pragma unroll
    for (int j = 0; j < K; ++j) dot[j] = 0.f;
    if (t < p.T) {
      const TokenPairs pair(p.pos, p.w, p.T, p.k, p.S, p.y_rows, t);
      for (int c = first * 512 + lane * 8; c < end; c += span) {  // (whole waves leave)
        Raw8<O> d;
        load_raw((const O*)p.dout + (size_t)t * p.ld_dout, c, p.cols, d);
        settle(d, c, p.cols);
        float block_max = 0.f;
        if (p.q) {
#pragma unroll
          for (int i = 0; i < 8; ++i) block_max = max_abs(block_max, d[i]);
          block_max = max16(block_max);
        }
        auto rows = [&](const Pair& a) {
          if (a.pos < 0) return;
          float o[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] = a.w * d[i];
          clear_beyond(o, c, p.cols);
          if (p.dy) store_cols((Y*)p.dy + (size_t)a.pos * p.ld_dy, c, p.cols, o);
          if (p.q) store_block(o, fmaxf(fabsf(a.w) * block_max, p.q_eps), c, p.cols, p.q + (size_t)a.pos * p.ldq, p.scale + (size_t)a.pos * p.ld_s);
        };
#pragma unroll
        for (int j0 = 0; j0 < K; j0 += NB) {
          if (j0 >= p.k) continue;
          Raw8<Y> v[NB];
          if (dots) {
#pragma unroll
            for (int u = 0; u < NB; ++u)  // (a row of any pair beyond the last, or without a position)
              load_raw((const Y*)p.y + (size_t)max(pair[min(j0 + u, p.k - 1)].pos, 0) * p.ldy, c, p.cols, v[u]);
          }
          if (p.dy || p.q) {
#pragma unroll
            for (int u = 0; u < NB; ++u)
              if (j0 + u < p.k) rows(pair[j0 + u]);
          }
          if (dots) {
#pragma unroll
            for (int u = 0; u < NB; ++u) {
              settle(v[u], c, p.cols);
              float s = 0.f;
#pragma unroll
              for (int i = 0; i < 8; ++i) s = fmaf(d[i], v[u][i], s);
              dot[j0 + u] += j0 + u < p.k && pair[j0 + u].pos >= 0 ? s : 0.f;
            }
          }
        }
        if (p.dy || p.q)
          for (int j = p.k; j < pairs; ++j) rows(pair[j]);
      }
    }
    if (p.dw) {
#pragma unroll
      for (int j = 0; j < K; ++j)
        if (j < p.k) {
          const float s = lanes_reduce<64, AddOp>(dot[j]);
          if (lane == 0) part[turn][wave][j] = s;
        }
      __syncthreads();
      if (t < p.T && first == 0 && lane < p.k) {
        float s = 0.f;
        for (int i = 0; i < 1 << share; ++i) s += part[turn][wave + i][lane];
        p.dw[(size_t)t * p.k + lane] = s;
      }
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
  const bool wide = p.T <= 256 && p.cols > 2048;
  const int share = wide ? 4 : p.cols <= 512 ? 0 : p.cols <= 1024 ? 1 : 2, per = wide ? 1 : 4 >> share;
  const uint32_t blocks = ((uint32_t)p.T + per - 1) / per;
  launch_timed("combine_grad", p.k <= 8 ? combine_grad_kernel<8, Y, O> : combine_grad_kernel<MIRA_MAX_TOPK, Y, O>,
               dim3(blocks < kMaxGrid ? blocks : kMaxGrid), dim3(wide ? 1024 : 256), 0, st, p, share);
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
