// Gradient of SwiGLU: of act = silu(gate) up, x = [gate | up], with s = sigmoid(gate),
//   dgate = d up s (1 + gate (1 - s)),  dup = d gate s,
// as rows and as e4m3 with one scale per block of 1 x 128.  Memory bound: each value is
// read once, eight columns of gate, up and d to a lane, and both results leave from there.
// Where cols is no multiple of 128, e4m3 blocks do not line up between the halves: lanes
// then go by blocks of the result and read their three values for each half.
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
// below 2^-126, where s times the rest is still a normal number.
__device__ __forceinline__ void swiglu_grad(float g, float u, float d, float* dg, float* du) {
  const float log2e = 1.44269502162933349609375f, rest = 1.92596299112661746887e-8f;
  const float t = -g * log2e;
  const float r = -fmaf(g, rest, fmaf(g, log2e, t));
  float e = __builtin_amdgcn_exp2f(t);
  e = fabsf(t) < 128.f ? fmaf(e, r * 0.693147182464599609375f, e) : e;
  const float s4 = __builtin_amdgcn_rcpf(fmaf(e, 0.25f, 0.25f));
  const float off = e < INFINITY ? e * (s4 * 0.25f) : 1.f;  // 1 - s
  *dg = (s4 * fmaf(g, off, 1.f)) * 0.25f * (d * u);
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

// By blocks of the result.
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
