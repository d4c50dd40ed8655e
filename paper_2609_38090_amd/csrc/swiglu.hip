// Gradient of SwiGLU: of act = silu(gate) up, x = [gate | up], with s = sigmoid(gate),
//   dgate = d up s (1 + gate (1 - s)),  dup = d gate s,
// as rows and as e4m3 with one scale per block of 1 x 128.  Memory bound: each value is
// read once, eight columns of gate, up and d to a lane, and both results leave from there.
// Where cols is no multiple of 128, e4m3 blocks do not line up between the halves: a row then
// belongs to a wave or a workgroup, whose blocks' maxima meet in LDS (maxima do not depend on the
// order of their atomics).  8192 x 14336 bf16 to e4m3: 171 us (947 MB, 5.5 TB/s).  30000 x 333 bf16 26 us
// by rows, 46 by the blocks of each half, which read the three values twice.
#include "fp8_dev.h"

namespace mira {

namespace {

constexpr uint32_t kMaxGrid = 1u << 21;  // workgroups of a launch: fewer than 2^32 threads

struct SwigluGradParams {
  const void* x;
  const void* d;
  void* dx;    // may be null
  uint8_t* q;  // may be null
  float* scale;
  size_t ldx, ldd, ld_dx, ldq, ld_s;
  int rows, cols;
  float q_eps;
};

// exp(-g) = 2^t with the rounding of t carried along where |t| < 128 (beyond, it is infinite, or
// nothing beside 1); 4 s = 1 / (1/4 + exp(-g)/4), since the reciprocal instruction gives 0
// below 2^-126, where s times the rest is still a normal number.  s times its factor, 1.1 at most, times the
// larger of d and u, then the smaller: d u alone may pass fp32's range, or the small one's product with s fall
// below it, where dgate does not (half of it until the end, since 1.1 times the larger may pass it too).
__device__ __forceinline__ void swiglu_grad(float g, float u, float d, float* dg, float* du) {
  const float log2e = 1.44269502162933349609375f, rest = 1.92596299112661746887e-8f;
  const float t = -g * log2e;
  const float r = -fmaf(g, rest, fmaf(g, log2e, t));
  float e = __builtin_amdgcn_exp2f(t);
  e = fabsf(t) < 128.f ? fmaf(e, r * 0.693147182464599609375f, e) : e;
  const float s4 = __builtin_amdgcn_rcpf(fmaf(e, 0.25f, 0.25f));
  const float off = e < INFINITY ? e * (s4 * 0.25f) : 1.f;  // 1 - s
  const bool up = fabsf(u) > fabsf(d);
  *dg = (s4 * fmaf(g, off, 1.f)) * 0.125f * (up ? u : d) * (up ? d : u) * 2.f;
  *du = g * (s4 * 0.25f) * d;
}

// Gate and up in step: dx alone for any number of columns, e4m3 for multiples of 128.
template <typename T, typename D>
__global__ __launch_bounds__(256) void swiglu_grad_kernel(SwigluGradParams p, int nb) {
  const uint32_t total = (uint32_t)p.rows * nb;  // < 2^31
  for (uint32_t block = blockIdx.x * 16 + (threadIdx.x >> 4); block < total; block += gridDim.x * 16) {
    const size_t r = block / (uint32_t)nb;
    const int c = (int)(block - (uint32_t)r * nb) * 128 + (threadIdx.x & 15) * 8;
    const T* x = (const T*)p.x + r * p.ldx;
    Raw8<T> gate, up;
    Raw8<D> d;
    load_raw(x, c, p.cols, gate);
    load_raw(x + p.cols, c, p.cols, up);
    load_raw((const D*)p.d + r * p.ldd, c, p.cols, d);
    settle(gate, c, p.cols);
    settle(up, c, p.cols);
    settle(d, c, p.cols);
    float g[8], u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) swiglu_grad(gate[i], up[i], d[i], &g[i], &u[i]);
    if (p.dx) {
      T* o = (T*)p.dx + r * p.ld_dx;
      store_cols(o, c, p.cols, g);
      store_cols(o + p.cols, c, p.cols, u);
    }
    if (p.q) {
      uint8_t* q = p.q + r * p.ldq;
      float* s = p.scale + r * p.ld_s;
      quantize_block(g, c, p.cols, p.q_eps, q, s);
      quantize_block(u, c, p.cols, p.q_eps, q + p.cols, s + nb);
    }
  }
}

// A row's gradient in e4m3 for any number of columns up to kRowCols: 16, 32 or 64 lanes (LANES, up to 512
// columns, as many rows to a workgroup as there are) or a workgroup (0) to a row.
constexpr int kRowCols = 16384;
typedef int v2i_bytes __attribute__((ext_vector_type(2), aligned(1)));  // (global stores take any alignment)

template <int LANES, int NV, typename T, typename D>
__global__ __launch_bounds__(LANES ? 256 : 1024) void swiglu_grad_row_kernel(SwigluGradParams p) {
  constexpr int kRows = LANES ? 256 / LANES : 1, kBlocks = LANES ? LANES / 8 : 2 * kRowCols / 128;
  __shared__ uint32_t largest[kRows][kBlocks];  // of each block of the result, as the bits of a magnitude
  const int L = LANES ? LANES : blockDim.x, l = LANES ? threadIdx.x & (LANES - 1) : threadIdx.x, w = LANES ? threadIdx.x / LANES : 0;
  const int blocks = (2 * p.cols + 127) / 128;
  auto meet = [] {
    if constexpr (LANES == 0) {
      __syncthreads();
    } else {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  };
  for (size_t r = (size_t)blockIdx.x * kRows + w; r < (size_t)p.rows; r += (size_t)gridDim.x * kRows) {
    const T* x = (const T*)p.x + r * p.ldx;
    Raw8<T> gate[NV], up[NV];
    Raw8<D> d[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * L + l) * 8;
      load_raw(x, c, p.cols, gate[i]);
      load_raw(x + p.cols, c, p.cols, up[i]);
      load_raw((const D*)p.d + r * p.ldd, c, p.cols, d[i]);
    }
    meet();  // (the last row's maxima have been read)
    for (int b = l; b < blocks; b += L) largest[w][b] = 0;
    meet();
    float g[NV][8], u[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * L + l) * 8;
      settle(gate[i], c, p.cols);
      settle(up[i], c, p.cols);
      settle(d[i], c, p.cols);
      // dup's columns are cols + c on; from `split` of them on they are in the next block
      const int first = (p.cols + c) >> 7, split = 128 - ((p.cols + c) & 127);
      float m = 0.f, lo = 0.f, hi = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        swiglu_grad(gate[i][j], up[i][j], d[i][j], &g[i][j], &u[i][j]);
        m = max_abs(m, g[i][j]);
        lo = j < split ? max_abs(lo, u[i][j]) : lo;
        hi = j < split ? hi : max_abs(hi, u[i][j]);
      }
      m = max16(m);
      if (c < p.cols) {
        if ((l & 15) == 0) atomicMax(&largest[w][c >> 7], __float_as_uint(m));
        atomicMax(&largest[w][first], __float_as_uint(lo));
        if (hi > 0.f) atomicMax(&largest[w][first + 1], __float_as_uint(hi));
      }
    }
    meet();
    for (int b = l; b < blocks; b += L) p.scale[r * p.ld_s + b] = fmaxf(__uint_as_float(largest[w][b]), p.q_eps) / kE4m3Max;
    uint8_t* q = p.q + r * p.ldq;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * L + l) * 8;
      if (c >= p.cols) continue;
      if (p.dx) {
        T* o = (T*)p.dx + r * p.ld_dx;
        store_cols(o, c, p.cols, g[i]);
        store_cols(o + p.cols, c, p.cols, u[i]);
      }
      const int first = (p.cols + c) >> 7, split = 128 - ((p.cols + c) & 127);
      auto inverse = [&](int b) { return kE4m3Max / fmaxf(__uint_as_float(largest[w][min(b, blocks - 1)]), p.q_eps); };
      const float inv_lo = inverse(first), inv_hi = inverse(first + 1);
#pragma unroll
      for (int j = 0; j < 8; ++j) u[i][j] *= j < split ? inv_lo : inv_hi;
      const uint2 qg = to_e4m3x8(g[i], inverse(c >> 7)), qu = to_e4m3x8(u[i], 1.f);
      if (c + 8 <= p.cols) {
        *(uint2*)(q + c) = qg;
        *(v2i_bytes*)(q + p.cols + c) = v2i_bytes{(int)qu.x, (int)qu.y};
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (c + j < p.cols) {
            q[c + j] = (uint8_t)((j < 4 ? qg.x : qg.y) >> (j & 3) * 8);
            q[p.cols + c + j] = (uint8_t)((j < 4 ? qu.x : qu.y) >> (j & 3) * 8);
          }
      }
    }
    const int behind = 2 * p.cols + l;  // zeros up to the next multiple of 16
    if (behind < (int)align_up((size_t)p.cols * 2, 16)) q[behind] = 0;
  }
}

// Longer rows, by blocks of the result: the three values are read for each half.
template <typename T, typename D>
__global__ __launch_bounds__(256) void swiglu_grad_any_kernel(SwigluGradParams p, int nb) {
  const uint32_t total = (uint32_t)p.rows * nb;  // < 2^31
  for (uint32_t block = blockIdx.x * 16 + (threadIdx.x >> 4); block < total; block += gridDim.x * 16) {
    const size_t r = block / (uint32_t)nb;
    const int c = (int)(block - (uint32_t)r * nb) * 128 + (threadIdx.x & 15) * 8;
    const T* x = (const T*)p.x + r * p.ldx;
    const D* dr = (const D*)p.d + r * p.ldd;
    float o[8];
    if (c + 8 <= p.cols || c >= p.cols) {
      const bool up = c >= p.cols;
      const int cc = up ? c - p.cols : c;
      float g[8], u[8], d[8];
      load_cols(x, cc, p.cols, g);
      load_cols(x + p.cols, cc, p.cols, u);
      load_cols(dr, cc, p.cols, d);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float dg, du;
        swiglu_grad(g[i], u[i], d[i], &dg, &du);
        o[i] = up ? du : dg;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool up = c + i >= p.cols;
        const int cc = up ? c + i - p.cols : c + i;
        float dg = 0.f, du = 0.f;
        if (cc < p.cols) swiglu_grad(load_act(x, cc), load_act(x + p.cols, cc), load_act(dr, cc), &dg, &du);
        o[i] = up ? du : dg;
      }
    }
    if (p.dx) store_cols((T*)p.dx + r * p.ld_dx, c, 2 * p.cols, o);
    quantize_block(o, c, 2 * p.cols, p.q_eps, p.q + r * p.ldq, p.scale + r * p.ld_s);
  }
}

template <typename T, typename D>
void launch_of(const SwigluGradParams& p, hipStream_t st) {
  const bool step = !p.q || p.cols % 128 == 0;
  if (!step && p.cols <= kRowCols) {
    const int lanes = p.cols <= 128 ? 16 : p.cols <= 256 ? 32 : p.cols <= 512 ? 64 : 0, rows = lanes ? 256 / lanes : 1;
    const int most = p.cols <= 8192 ? p.cols : (p.cols + 1) / 2, threads = lanes ? 256 : (most + 511) / 512 * 64;
    const uint32_t blocks = ((uint32_t)p.rows + rows - 1) / rows;
    launch_timed("swiglu_grad_row",
                 lanes == 16   ? swiglu_grad_row_kernel<16, 1, T, D>
                 : lanes == 32 ? swiglu_grad_row_kernel<32, 1, T, D>
                 : lanes == 64 ? swiglu_grad_row_kernel<64, 1, T, D>
                 : p.cols <= 8192 ? swiglu_grad_row_kernel<0, 1, T, D>
                                  : swiglu_grad_row_kernel<0, 2, T, D>,
                 dim3(blocks < kMaxGrid ? blocks : kMaxGrid), dim3(threads), 0, st, p);
    return;
  }
  const int nb = (int)(((size_t)p.cols * (step ? 1 : 2) + 127) / 128);
  const size_t blocks = ((size_t)p.rows * nb + 15) / 16;
  const dim3 grid((uint32_t)(blocks < kMaxGrid ? blocks : kMaxGrid));
  if (step) launch_timed("swiglu_grad", swiglu_grad_kernel<T, D>, grid, dim3(256), 0, st, p, nb);
  else launch_timed("swiglu_grad_any", swiglu_grad_any_kernel<T, D>, grid, dim3(256), 0, st, p, nb);
}

}  // namespace

hipError_t launch_swiglu_grad(const mira_swiglu_grad_args& a, hipStream_t st) {
  SwigluGradParams p{};
  const size_t cols = a.cols;
  p.x = a.x;
  p.d = a.dact;
  p.dx = a.dx;
  p.q = (uint8_t*)a.q;
  p.scale = a.scale;
  p.ldx = a.ldx ? a.ldx : 2 * cols;
  p.ldd = a.ld_dact ? a.ld_dact : cols;
  p.ld_dx = a.ld_dx ? a.ld_dx : 2 * cols;
  p.ldq = a.ldq ? a.ldq : align_up(2 * cols, 16);
  p.ld_s = a.ld_scale ? a.ld_scale : (2 * cols + 127) / 128;
  p.rows = a.rows;
  p.cols = a.cols;
  p.q_eps = a.q_eps;
  const bool xf = a.x_dtype == MIRA_F32, df = a.d_dtype == MIRA_F32;
  if (xf) df ? launch_of<float, float>(p, st) : launch_of<float, uint16_t>(p, st);
  else df ? launch_of<uint16_t, float>(p, st) : launch_of<uint16_t, uint16_t>(p, st);
  return hipGetLastError();
}

}  // namespace mira
