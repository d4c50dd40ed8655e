// Root-mean-square norm of h = x + residual with an output in e4m3, and its gradient.
//   y = h r w,  r = (mean of h^2 + eps)^-1/2;
//   dx = dsum + r (g - n mean(n g)),  g = dy w,  n = h r;   dweight = sum over rows of dy n.
// Memory bound: a row is read once into registers, eight consecutive columns to a lane
// (16 bytes of bf16; 16 lanes hold a block of 128 that shares a scale), its sums are taken
// across the lanes, and every output is written from there.  A row is shared by as many lanes
// as hold it at eight values each (sixteen above 8192 columns): 16, 32 or a wave, a workgroup of its own from
// two waves on; rows of more than 16384 are read twice.  The gradient of the weight is summed in
// registers over the rows that a workgroup walks, then over workgroups in order.  4096 x 4096 bf16 with
// residual, y and e4m3 30 us (151 MB, 5.0 TB/s; a copy of 1 GB reaches 5.2); the gradient of 16384 x 4096
// 102 us (537 MB, 5.3 TB/s).
#include "fp8_dev.h"

namespace mira {

namespace {

constexpr int kLongParts = 64;   // parts of the rows, for rows that registers do not hold
constexpr int kRegCols = 16384;  // columns of a row that registers hold
constexpr uint32_t kMaxGrid = 1u << 21;  // workgroups of a launch: fewer than 2^32 threads

// A row's sum of squares beyond fp32's range is taken of the row times 2^-80 (the mean of
// 2^24 squares of fp32's largest values fits then).
constexpr float kDown = 8.271806125530276748714e-25f;

// Workgroups of one row have 128 to 1024 threads, those of several rows (16, 32 or 64 lanes each) 256: waves
// of one row meet at barriers, which rows of one workgroup could not do apart.
int row_lanes(int cols) { return cols <= 128 ? 16 : cols <= 256 ? 32 : cols <= 512 ? 64 : 0; }  // 0: the workgroup
int row_threads(int cols) {
  if (cols <= 512) return 256;
  const int n = cols <= 8192 ? cols : (cols + 1) / 2;
  return (n + 511) / 512 * 64;
}

// Workgroups that sum the gradient of the weight: as many to each CU, of no more than 1024 threads together
// (17879 x 2787 bf16 in 682, which some CUs had two and some three of, 126 us, in 512 90; 6000 x 7168
// in 292 102 us, in 256 70; with up to 1280 threads to a CU 117 and 70).
int parts_of(int threads) { return 256 * (1024 / threads); }

struct NormParams {
  const void* x;
  const void* residual;  // may be null
  const void* w;
  void* sum;             // may be null
  void* y;               // may be null
  uint8_t* q;            // may be null
  float* scale;
  size_t ldx, ld_res, ld_sum, ldy, ldq, ld_s;
  int rows, cols;
  bool w_f32, y_f32;
  float eps, q_eps;
};

struct NormGradParams {
  const void* dy;
  const void* dsum;  // may be null
  const void* h;
  const void* w;
  void* dx;          // may be null
  float* partial;    // [workgroups][cols]
  float* rstd;       // [rows] (long rows)
  size_t ld_dy, ld_dsum, ld_h, ld_dx;
  int rows, cols;
  bool w_f32, y_f32;
  float eps;
};

// Eight values of a row that is fp32 or bf16.
__device__ __forceinline__ void load8(const void* p, size_t row_at, bool f32, int c, int cols, float (&v)[8]) {
  if (f32) load_cols((const float*)p + row_at, c, cols, v);
  else load_cols((const uint16_t*)p + row_at, c, cols, v);
}

// Sum over the threads of a row, in all of them: LANES of them, or (0) the workgroup, whose waves meet in
// LDS.  `turn` alternates between two sets of it, so that one barrier a sum suffices.
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float (*part)[16], int turn) {
  v = lanes_reduce<LANES ? LANES : 64, AddOp>(v);
  if constexpr (LANES == 0) {
    if ((threadIdx.x & 63) == 0) part[turn][threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
    for (int i = 0; i < (int)blockDim.x >> 6; ++i) v += part[turn][i];
  }
  return v;
}
// Two sums at once.
template <int LANES>
__device__ __forceinline__ void row_sum2(float& a, float& b, float2 (*part)[16], int turn) {
  a = lanes_reduce<LANES ? LANES : 64, AddOp>(a);
  b = lanes_reduce<LANES ? LANES : 64, AddOp>(b);
  if constexpr (LANES == 0) {
    if ((threadIdx.x & 63) == 0) part[turn][threadIdx.x >> 6] = float2{a, b};
    __syncthreads();
    a = b = 0.f;
    for (int i = 0; i < (int)blockDim.x >> 6; ++i) {
      a += part[turn][i].x;
      b += part[turn][i].y;
    }
  }
}

template <int LANES, int NV, typename T, typename W>
__global__ __launch_bounds__(LANES ? 256 : 1024) void rmsnorm_kernel(NormParams p) {
  constexpr int kRows = LANES ? 256 / LANES : 1;
  __shared__ float part[4][16];
  const int L = LANES ? LANES : blockDim.x, l = LANES ? threadIdx.x & (LANES - 1) : threadIdx.x, in_block = LANES ? threadIdx.x / LANES : 0;
  const float inv_cols = 1.f / (float)p.cols;
  int turn = 0;
  for (size_t r = (size_t)blockIdx.x * kRows + in_block; r < (size_t)p.rows; r += (size_t)gridDim.x * kRows) {
    const T* x = (const T*)p.x + r * p.ldx;
    float v[NV][8], ss = 0.f;
    Raw8<T> raw[NV], res[NV];
    Raw8<W> w[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) load_raw(x, (i * L + l) * 8, p.cols, raw[i]);
    if (p.residual) {
      const T* e = (const T*)p.residual + r * p.ld_res;
#pragma unroll
      for (int i = 0; i < NV; ++i) load_raw(e, (i * L + l) * 8, p.cols, res[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) load_raw((const W*)p.w, (i * L + l) * 8, p.cols, w[i]);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      settle(raw[i], (i * L + l) * 8, p.cols);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = raw[i][j];
    }
    if (p.residual) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        settle(res[i], (i * L + l) * 8, p.cols);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = held(v[i][j] + res[i][j], x);
      }
    }
    if (p.sum) {
#pragma unroll
      for (int i = 0; i < NV; ++i) store_cols((T*)p.sum + r * p.ld_sum, (i * L + l) * 8, p.cols, v[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) ss = fmaf(v[i][j], v[i][j], ss);
    ss = row_sum<LANES>(ss, part, turn & 1);
    float rs;
    if (ss <= 3.4028234e38f || ss != ss) {
      rs = __builtin_amdgcn_rsqf(fmaf(ss, inv_cols, p.eps));
    } else {  // (the whole row's threads)
      ss = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[i][j] *= kDown;
          ss = fmaf(v[i][j], v[i][j], ss);
        }
      ss = row_sum<LANES>(ss, part, 2 + (turn & 1));
      rs = __builtin_amdgcn_rsqf(fmaf(ss, inv_cols, p.eps * kDown * kDown));
    }
    ++turn;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * L + l) * 8;
      settle(w[i], c, p.cols);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = v[i][j] * rs * w[i][j];
      if (p.y) {
        if (p.y_f32) store_cols((float*)p.y + r * p.ldy, c, p.cols, v[i]);
        else store_cols((uint16_t*)p.y + r * p.ldy, c, p.cols, v[i]);
      }
      if (p.q) quantize_block(v[i], c, p.cols, p.q_eps, p.q + r * p.ldq, p.scale + r * p.ld_s);
    }
  }
}

// Rows that registers do not hold: a workgroup walks its row for the sum, then again
// (from sum, where that is written: it may be x's or the residual's own memory, and a
// thread meets its own columns only).
template <typename T>
__global__ __launch_bounds__(1024) void rmsnorm_long_kernel(NormParams p) {
  __shared__ float part[4][16];
  const int end = (int)align_up((size_t)p.cols, 8192);  // whole waves take every step
  const float inv_cols = 1.f / (float)p.cols;
  int turn = 0;
  for (size_t r = blockIdx.x; r < (size_t)p.rows; r += gridDim.x) {
    const T* x = (const T*)p.x + r * p.ldx;
    const T* e = p.residual ? (const T*)p.residual + r * p.ld_res : nullptr;
    auto row = [&](int c, float (&v)[8]) {
      load_cols(x, c, p.cols, v);
      if (e) {
        float o[8];
        load_cols(e, c, p.cols, o);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = held(v[j] + o[j], x);
      }
    };
    float ss = 0.f, down = 0.f;
    for (int c = threadIdx.x * 8; c < end; c += 8192) {
      float v[8];
      row(c, v);
      if (p.sum) store_cols((T*)p.sum + r * p.ld_sum, c, p.cols, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        ss = fmaf(v[j], v[j], ss);
        const float d = v[j] * kDown;
        down = fmaf(d, d, down);
      }
    }
    ss = row_sum<0>(ss, part, turn & 1);
    down = row_sum<0>(down, part, 2 + (turn & 1));
    ++turn;
    const bool far = ss > 3.4028234e38f;
    const float rs = __builtin_amdgcn_rsqf(far ? fmaf(down, inv_cols, p.eps * kDown * kDown) : fmaf(ss, inv_cols, p.eps)), pre = far ? kDown : 1.f;
    for (int c = threadIdx.x * 8; c < end; c += 8192) {
      float v[8], w[8];
      if (p.sum) load_cols((const T*)p.sum + r * p.ld_sum, c, p.cols, v);
      else row(c, v);
      load8(p.w, 0, p.w_f32, c, p.cols, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = v[j] * pre * rs * w[j];
      if (p.y) {
        if (p.y_f32) store_cols((float*)p.y + r * p.ldy, c, p.cols, v);
        else store_cols((uint16_t*)p.y + r * p.ldy, c, p.cols, v);
      }
      if (p.q) quantize_block(v, c, p.cols, p.q_eps, p.q + r * p.ldq, p.scale + r * p.ld_s);
    }
  }
}

// A row's gradient: the sums of h^2 and of h dy w, of h times 2^-80 where the first passes
// fp32's range; r, and the mean of n g.
struct RowGrad {
  float pre, rs, inner;  // n = h pre rs
};
template <int LANES, int NV, typename T, typename D, typename W>
__device__ __forceinline__ RowGrad grad_sums(const Raw8<T> (&h)[NV], const Raw8<D> (&d)[NV], W weights, float eps, float inv_cols,
                                             float2 (*part)[16], int turn) {
  RowGrad o;
  o.pre = 1.f;
  float ss, hg;
  auto sums = [&](int set) {
    ss = 0.f, hg = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float w[8];
      weights(i, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float v = h[i][j] * o.pre;
        ss = fmaf(v, v, ss);
        hg = fmaf(v, d[i][j] * w[j], hg);
      }
    }
    row_sum2<LANES>(ss, hg, part, set);
  };
  sums(turn & 1);
  if (ss > 3.4028234e38f) {  // (the whole row's threads)
    o.pre = kDown;
    sums(2 + (turn & 1));
    o.rs = __builtin_amdgcn_rsqf(fmaf(ss, inv_cols, eps * kDown * kDown));
  } else {
    o.rs = __builtin_amdgcn_rsqf(fmaf(ss, inv_cols, eps));
  }
  o.inner = o.rs * hg * inv_cols;
  return o;
}

template <int LANES, int NV, bool DW, typename T, typename D>
__global__ __launch_bounds__(LANES ? 256 : 1024) void rmsnorm_grad_kernel(NormGradParams p) {
  constexpr int kRows = LANES ? 256 / LANES : 1;
  __shared__ float2 part[4][16];
  const int L = LANES ? LANES : blockDim.x, l = LANES ? threadIdx.x & (LANES - 1) : threadIdx.x, in_block = LANES ? threadIdx.x / LANES : 0;
  const float inv_cols = 1.f / (float)p.cols;
  float held_w[8], acc[NV][8];
  load8(p.w, 0, p.w_f32, l * 8, p.cols, held_w);
  auto weights = [&](int i, float (&w)[8]) {  // (of two in a row, registers have no room for the second)
    if (i == 0) {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = held_w[j];
    } else {
      const void* again = p.w;  // (a load of its own in every row, not one kept through them)
      asm volatile("" : "+s"(again));
      load8(again, 0, p.w_f32, (i * L + l) * 8, p.cols, w);
    }
  };
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = 0.f;
  int turn = 0;
  for (size_t r = (size_t)blockIdx.x * kRows + in_block; r < (size_t)p.rows; r += (size_t)gridDim.x * kRows, ++turn) {
    Raw8<T> h[NV], s[NV];
    Raw8<D> d[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * L + l) * 8;
      load_raw((const T*)p.h + r * p.ld_h, c, p.cols, h[i]);
      load_raw((const D*)p.dy + r * p.ld_dy, c, p.cols, d[i]);
    }
    if (p.dsum) {
#pragma unroll
      for (int i = 0; i < NV; ++i) load_raw((const T*)p.dsum + r * p.ld_dsum, (i * L + l) * 8, p.cols, s[i]);
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) s[i].zero();
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * L + l) * 8;
      settle(h[i], c, p.cols);
      settle(d[i], c, p.cols);
      settle(s[i], c, p.cols);
    }
    const RowGrad o = grad_sums<LANES, NV>(h, d, weights, p.eps, inv_cols, part, turn);
    const float out_scale = o.rs * o.pre;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float dx[8], w[8];
      weights(i, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float n = h[i][j] * o.pre * o.rs;
        if constexpr (DW) acc[i][j] = fmaf(d[i][j], n, acc[i][j]);
        dx[j] = fmaf(out_scale, d[i][j] * w[j] - n * o.inner, s[i][j]);
      }
      if (p.dx) store_cols((T*)p.dx + r * p.ld_dx, (i * L + l) * 8, p.cols, dx);
    }
  }
  if constexpr (DW) {
    float* out = p.partial + (size_t)blockIdx.x * p.cols;
    if constexpr (LANES == 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) store_cols(out, (i * L + l) * 8, p.cols, acc[i]);
    } else {
      __shared__ float rows_acc[kRows][LANES * 8];
#pragma unroll
      for (int j = 0; j < 8; ++j) rows_acc[in_block][l * 8 + j] = acc[0][j];
      __syncthreads();
      for (int c = threadIdx.x; c < p.cols; c += 256) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < kRows; ++i) s += rows_acc[i][c];
        out[c] = s;
      }
    }
  }
}

// Rows that registers do not hold, for dx and r.
template <typename T>
__global__ __launch_bounds__(1024) void rmsnorm_grad_long_kernel(NormGradParams p) {
  __shared__ float part[8][16];
  const int end = (int)align_up((size_t)p.cols, 8192);
  const float inv_cols = 1.f / (float)p.cols;
  int turn = 0;
  for (size_t r = blockIdx.x; r < (size_t)p.rows; r += gridDim.x, ++turn) {
    auto at = [&](int c, float (&h)[8], float (&g)[8]) {
      float w[8];
      load_cols((const T*)p.h + r * p.ld_h, c, p.cols, h);
      load8(p.dy, r * p.ld_dy, p.y_f32, c, p.cols, g);
      load8(p.w, 0, p.w_f32, c, p.cols, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] *= w[j];
    };
    float ss = 0.f, hg = 0.f, ds = 0.f, dg = 0.f;
    for (int c = threadIdx.x * 8; c < end; c += 8192) {
      float h[8], g[8];
      at(c, h, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = h[j] * kDown;
        ss = fmaf(h[j], h[j], ss);
        hg = fmaf(h[j], g[j], hg);
        ds = fmaf(d, d, ds);
        dg = fmaf(d, g[j], dg);
      }
    }
    const int b = (turn & 1) * 4;
    ss = row_sum<0>(ss, part, b);
    hg = row_sum<0>(hg, part, b + 1);
    ds = row_sum<0>(ds, part, b + 2);
    dg = row_sum<0>(dg, part, b + 3);
    const bool far = ss > 3.4028234e38f;
    const float rs = __builtin_amdgcn_rsqf(far ? fmaf(ds, inv_cols, p.eps * kDown * kDown) : fmaf(ss, inv_cols, p.eps)), pre = far ? kDown : 1.f;
    const float inner = rs * (far ? dg : hg) * inv_cols;
    if (p.rstd && threadIdx.x == 0) p.rstd[r] = far ? -rs : rs;  // the sign says that rows are scaled first
    if (!p.dx) continue;
    for (int c = threadIdx.x * 8; c < end; c += 8192) {
      float h[8], g[8], o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      at(c, h, g);
      if (p.dsum) load_cols((const T*)p.dsum + r * p.ld_dsum, c, p.cols, o);
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = fmaf(rs * pre, g[j] - h[j] * pre * rs * inner, o[j]);
      store_cols((T*)p.dx + r * p.ld_dx, c, p.cols, o);
    }
  }
}

// ... and a part of the rows for the gradient of 2048 columns of the weight.
template <typename T>
__global__ __launch_bounds__(256) void rmsnorm_grad_long_weight_kernel(NormGradParams p) {
  const int c = (blockIdx.x * 256 + threadIdx.x) * 8, n = gridDim.y;
  if (c >= p.cols) return;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (size_t r = blockIdx.y; r < (size_t)p.rows; r += n) {
    float h[8], d[8];
    load_cols((const T*)p.h + r * p.ld_h, c, p.cols, h);
    load8(p.dy, r * p.ld_dy, p.y_f32, c, p.cols, d);
    const float rs = p.rstd[r], pre = rs < 0.f ? kDown : 1.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = fmaf(d[j], h[j] * pre * fabsf(rs), acc[j]);
  }
  store_cols(p.partial + (size_t)blockIdx.y * p.cols, c, p.cols, acc);
}

// Sums the workgroups' parts in order: 32 columns to a workgroup, 32 threads to each 32nd of the parts.
__global__ __launch_bounds__(1024) void rmsnorm_weight_kernel(const float* __restrict__ partial, int parts, int cols,
                                                              float* __restrict__ dw) {
  __shared__ float sums[32][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
  float s = 0.f;
  if (c < cols) {
    const int lo = (int)((int64_t)parts * y / 32), hi = (int)((int64_t)parts * (y + 1) / 32);
#pragma unroll 8
    for (int i = lo; i < hi; ++i) s += partial[(size_t)i * cols + c];
  }
  sums[y][x] = s;
  __syncthreads();
  if (y == 0 && c < cols) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += sums[i][x];
    dw[c] = s;
  }
}

int rows_per_block(int cols) { return row_lanes(cols) ? 256 / row_lanes(cols) : 1; }

uint32_t row_grid(int rows, int per_block, uint32_t most) {
  const uint32_t n = ((uint32_t)rows + per_block - 1) / per_block;
  return n < most ? n : most;
}

template <typename T, typename W>
void launch_norm_of(const NormParams& p, hipStream_t st) {
  const int lanes = row_lanes(p.cols);
  if (p.cols > kRegCols)
    launch_timed("rmsnorm_long", rmsnorm_long_kernel<T>, dim3(row_grid(p.rows, 1, kMaxGrid)), dim3(1024), 0, st, p);
  else
    launch_timed("rmsnorm",
                 lanes == 16   ? rmsnorm_kernel<16, 1, T, W>
                 : lanes == 32 ? rmsnorm_kernel<32, 1, T, W>
                 : lanes == 64 ? rmsnorm_kernel<64, 1, T, W>
                 : p.cols <= 8192 ? rmsnorm_kernel<0, 1, T, W>
                                  : rmsnorm_kernel<0, 2, T, W>,
                 dim3(row_grid(p.rows, rows_per_block(p.cols), kMaxGrid)), dim3(row_threads(p.cols)), 0, st, p);
}

// Parts of the weight's gradient: two rows to a workgroup where there are not many for each (1201 x
// 2001 fp32: 12.7 us so, 14.2 with one, whose parts are as many bytes as the rows; 13.2 with three or four).
constexpr int kPartRows = 2;
// One workgroup writes the gradient itself where it has few rows in turn (us of three, four, five and six: 4096 bf16 5.6,
// 5.2, 5.9 and 6.8, 2000 fp32 four to six 6.1, 7.1 and 8.2, 8000 fp32 three and four 7.7 and 9.5, against 7.5 to
// 8.3 in two launches; 12510 columns four 16 against 8.8).
int one_part(int cols) { return cols <= 4096 ? 5 : cols <= 8192 ? 3 : 1; }
int parts_for(int rows, int cols, int per_block, int most) {
  const int few = (int)(((uint32_t)rows + per_block - 1) / per_block);  // one row after another
  if (few <= one_part(cols)) return min(few, 1);
  return min(most, max((few + kPartRows - 1) / kPartRows, min(few, 256)));
}

int grad_parts(int rows, int cols) {
  if (cols > kRegCols) return rows < kLongParts ? rows : kLongParts;
  return parts_for(rows, cols, rows_per_block(cols), parts_of(row_threads(cols)));
}

// Launches the rows' pass; returns the parts of the weight's gradient that it leaves.
template <bool DW, typename T, typename D>
int launch_grad(const NormGradParams& p, hipStream_t st) {
  const int lanes = row_lanes(p.cols);
  const uint32_t grid = DW ? (uint32_t)grad_parts(p.rows, p.cols) : row_grid(p.rows, rows_per_block(p.cols), kMaxGrid);
  launch_timed("rmsnorm_grad",
               lanes == 16   ? rmsnorm_grad_kernel<16, 1, DW, T, D>
               : lanes == 32 ? rmsnorm_grad_kernel<32, 1, DW, T, D>
               : lanes == 64 ? rmsnorm_grad_kernel<64, 1, DW, T, D>
               : p.cols <= 8192 ? rmsnorm_grad_kernel<0, 1, DW, T, D>
                                : rmsnorm_grad_kernel<0, 2, DW, T, D>,
               dim3(grid), dim3(row_threads(p.cols)), 0, st, p);
  return (int)grid;
}

template <typename T>
int launch_grad_of(const NormGradParams& p, bool dw, hipStream_t st) {
  if (p.cols <= kRegCols) {
    if (p.y_f32) return dw ? launch_grad<true, T, float>(p, st) : launch_grad<false, T, float>(p, st);
    return dw ? launch_grad<true, T, uint16_t>(p, st) : launch_grad<false, T, uint16_t>(p, st);
  }
  launch_timed("rmsnorm_grad_long", rmsnorm_grad_long_kernel<T>, dim3(row_grid(p.rows, 1, kMaxGrid)), dim3(1024), 0, st, p);
  const int parts = grad_parts(p.rows, p.cols);
  if (dw)
    launch_timed("rmsnorm_grad_long_weight", rmsnorm_grad_long_weight_kernel<T>, dim3((p.cols + 2047) / 2048, parts), dim3(256), 0, st, p);
  return parts;
}

size_t or_dense(uint64_t ld, size_t dense) { return ld ? ld : dense; }

}  // namespace

hipError_t launch_rmsnorm(const mira_rmsnorm_args& a, hipStream_t st) {
  NormParams p{};
  const size_t cols = a.cols;
  p.x = a.x;
  p.residual = a.residual;
  p.w = a.weight;
  p.sum = a.sum;
  p.y = a.y;
  p.q = (uint8_t*)a.q;
  p.scale = a.scale;
  p.ldx = or_dense(a.ldx, cols);
  p.ld_res = or_dense(a.ld_res, cols);
  p.ld_sum = or_dense(a.ld_sum, cols);
  p.ldy = or_dense(a.ldy, cols);
  p.ldq = or_dense(a.ldq, align_up(cols, 16));
  p.ld_s = or_dense(a.ld_scale, (cols + 127) / 128);
  p.rows = a.rows;
  p.cols = a.cols;
  p.w_f32 = a.w_dtype == MIRA_F32;
  p.y_f32 = a.y_dtype == MIRA_F32;
  p.eps = a.eps;
  p.q_eps = a.q_eps;
  if (a.x_dtype == MIRA_F32) p.w_f32 ? launch_norm_of<float, float>(p, st) : launch_norm_of<float, uint16_t>(p, st);
  else p.w_f32 ? launch_norm_of<uint16_t, float>(p, st) : launch_norm_of<uint16_t, uint16_t>(p, st);
  return hipGetLastError();
}

size_t rmsnorm_grad_ws_bytes(int rows, int cols) {
  const size_t rstd = cols > kRegCols ? align_up((size_t)rows * 4, 256) : 0;
  return align_up(rstd + (size_t)grad_parts(rows, cols) * cols * 4, 256) + 256;
}

hipError_t launch_rmsnorm_grad(const mira_rmsnorm_grad_args& a, hipStream_t st) {
  NormGradParams p{};
  const size_t cols = a.cols;
  p.dy = a.dy;
  p.dsum = a.dsum;
  p.h = a.h;
  p.w = a.weight;
  p.dx = a.dx;
  p.ld_dy = or_dense(a.ld_dy, cols);
  p.ld_dsum = or_dense(a.ld_dsum, cols);
  p.ld_h = or_dense(a.ld_h, cols);
  p.ld_dx = or_dense(a.ld_dx, cols);
  p.rows = a.rows;
  p.cols = a.cols;
  p.w_f32 = a.w_dtype == MIRA_F32;
  p.y_f32 = a.y_dtype == MIRA_F32;
  p.eps = a.eps;
  const bool dw = a.dweight != nullptr;
  if (dw) {
    const bool is_long = a.cols > kRegCols;
    p.rstd = is_long ? (float*)a.workspace : nullptr;
    p.partial = (float*)((char*)a.workspace + (is_long ? align_up((size_t)a.rows * 4, 256) : 0));
    if (grad_parts(a.rows, a.cols) == 1) p.partial = a.dweight;
  }
  int parts = 0;
  if (a.rows > 0) parts = a.x_dtype == MIRA_F32 ? launch_grad_of<float>(p, dw, st) : launch_grad_of<uint16_t>(p, dw, st);
  if (dw && parts != 1)
    launch_timed("rmsnorm_weight", rmsnorm_weight_kernel, dim3((a.cols + 31) / 32), dim3(1024), 0, st, (const float*)p.partial,
                 parts, a.cols, a.dweight);
  return hipGetLastError();
}

}  // namespace mira
