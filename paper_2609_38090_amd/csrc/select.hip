// Selection of experts from logits, the order of the (token, expert) pairs, and
// the gradient of the weights.
//
// Selection: a wave takes a row, V consecutive experts to a lane, so that the lowest lane
// of equal values has the lowest expert.  Without a bias (and without sums of a group's two
// best) the logits themselves are compared, which is exact.  Otherwise c = s + bias is
// computed in fp32 with an error below `delta` (see margin_of); where two candidates of a
// step lie closer than their errors allow, the row is done again with c in 64 bits.
//
// Order: a chunk of tokens is a workgroup.  Each expert has a bit for every token of the
// chunk, so a pair's rank in its expert's list is a count of bits: no order of atomics
// decides anything.  Counts of all chunks are added up by a launch in between.
#include "device_util.h"
#include "mira_internal.h"

namespace mira {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kChunk = 256;     // most tokens of a chunk
constexpr int kWords = kChunk / 32;
constexpr float kTiny = 1e-20f;
constexpr int kMaxGrid = 1 << 21;  // workgroups of 256 threads: fewer than 2^32 in a launch

struct SelectParams {
  const void* logits;
  const float* bias;    // may be null
  const uint8_t* mask;  // may be null
  int32_t* idx;
  float* weight;        // may be null
  int32_t* counts;      // [chunks][G] workspace
  int32_t* totals;      // [G] workspace
  int32_t* counts_out;  // may be null, as the next three
  int32_t* offsets_out;
  int32_t* order;
  int32_t* pos;
  size_t ld;
  int T, E, k, S, groups, top_groups, best, chunk, chunks;
  bool sigmoid, renorm, place;
  float scale;
};

__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ float wave_best(float v) { return lanes_reduce<64, MaxOp>(v); }
__device__ __forceinline__ double wave_best(double v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = fmax(v, __shfl_xor(v, o, 64));
  return v;
}

// 1 / (1 + exp(-x)) without overflow, 4 steps.
__device__ __forceinline__ float sigmoid(float x) {
  const float e = exp_neg(-fabsf(x)), r = __builtin_amdgcn_rcpf(1.f + e);
  return x >= 0.f ? r : e * r;
}

// The selection proper: key[i] is the rank of expert V lane + i (-inf: not to be selected),
// gkey[i] its c for the groups' scores.  Lane j < k returns the j-th expert or -1.  With
// margins above 0, *close is set where they do not tell two candidates apart.
template <int V, typename F>
__device__ __forceinline__ int choose(const SelectParams& p, F (&key)[V], const F (&gkey)[V], F key_margin, F group_margin,
                                      F* scr, bool* close) {
  const int lane = threadIdx.x & 63;
  const F none = -(F)INFINITY;
  bool near = false;
  if (p.groups > 1) {
    const int size = p.E / p.groups;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (V * lane + i < p.E) scr[V * lane + i] = gkey[i];
    wave_sync();
    F score[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int g = lane + 64 * i;
      score[i] = none;
      if (g >= p.groups) continue;
      F b1 = none, b2 = none;
      for (int e = g * size; e < (g + 1) * size; ++e) {
        const F c = scr[e];
        b2 = c > b1 ? b1 : c > b2 ? c : b2;
        b1 = c > b1 ? c : b1;
      }
      score[i] = p.best == 2 && b2 != none ? b1 + b2 : b1;
    }
    wave_sync();
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (lane + 64 * i < p.groups) scr[lane + 64 * i] = score[i];
    wave_sync();
    bool keep[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int g = lane + 64 * i;
      keep[i] = false;
      if (g >= p.groups) continue;
      int before = 0;
      for (int h = 0; h < p.groups; ++h) {
        const F o = scr[h];
        before += o > score[i] || (o == score[i] && h < g);
        near |= h != g && o != none && fabs(o - score[i]) <= group_margin;
      }
      keep[i] = before < p.top_groups;
    }
    wave_sync();
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (lane + 64 * i < p.groups) scr[lane + 64 * i] = keep[i] ? (F)1 : (F)0;
    wave_sync();
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (V * lane + i < p.E && scr[(V * lane + i) / size] == (F)0) key[i] = none;
    wave_sync();
  }
  int mine = -1;
  for (int j = 0; j < p.k; ++j) {
    F b = key[0];
#pragma unroll
    for (int i = 1; i < V; ++i) b = key[i] > b ? key[i] : b;
    const F m = wave_best(b);
    if (m == none) break;
    const int who = __ffsll((unsigned long long)__ballot(b == m)) - 1;
    int at = 0;
#pragma unroll
    for (int i = V - 1; i >= 0; --i) at = key[i] == m ? i : at;
    const int e = __builtin_amdgcn_readlane(V * lane + at, who);
    if (lane == j) mine = e;
    if (lane == who) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i == at) key[i] = none;
    }
    if (key_margin >= (F)0) {
#pragma unroll
      for (int i = 0; i < V; ++i) near |= key[i] >= m - key_margin;
    }
  }
  *close = __ballot(near) != 0;
  return mine;
}

// One row by one wave.  Lane j < k returns the j-th expert (or -1) and its weight.
template <int V, typename T>
__device__ __forceinline__ int select_row(const SelectParams& p, int row, const float (&bias)[V], float bias_max, double* scr,
                                          float* weight) {
  const int lane = threadIdx.x & 63;
  *weight = 0.f;
  if (p.mask && !p.mask[row]) return -1;
  const T* x = (const T*)p.logits + (size_t)row * p.ld;
  float v[V], s[V];
  bool nan = false;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    v[i] = V * lane + i < p.E ? load_act(x, V * lane + i) : -INFINITY;
    nan |= v[i] != v[i];
  }
  float top = 1.f;  // the largest score
  float m = 0.f, sum = 1.f;
  if (p.sigmoid) {
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = sigmoid(v[i]);
  } else {
    m = v[0];
#pragma unroll
    for (int i = 1; i < V; ++i) m = fmaxf(m, v[i]);
    m = lanes_reduce<64, MaxOp>(m);
    nan |= m == INFINITY;
    m = m == -INFINITY ? 0.f : m;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      s[i] = exp_neg(v[i] - m);
      sum += s[i];
    }
    sum = lanes_reduce<64, AddOp>(sum);
    top = sum == 0.f ? 0.f : __builtin_amdgcn_rcpf(sum);
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] *= top;
  }
  nan = __ballot(nan) != 0;
  const bool sums = p.groups > 1 && p.best == 2;
  float key[V], gkey[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const bool can = v[i] > -INFINITY;  // (neither -inf nor NaN)
    const float c = p.bias ? s[i] + bias[i] : s[i];
    key[i] = !can ? -INFINITY : p.bias && !nan ? c : v[i];
    gkey[i] = !can ? -INFINITY : (p.bias || sums) && !nan ? c : v[i];
  }
  // An s is off by less than 2^-19 of the largest (softmax: 2 steps of exp, 10 additions, the
  // reciprocal and a product, 20 half steps in all; sigmoid: 8), c by the addition's half step
  // more; two of them, and a sum of two against another, by 2 and 4 times that (and its half step).
  const float delta = 0x1p-19f * top + 0x1p-22f * (top + bias_max);
  bool close;
  int e = choose<V, float>(p, key, gkey, p.bias && !nan ? 2.f * delta : -1.f, (p.bias || sums) && !nan ? 4.5f * delta : -1.f, (float*)scr,
                           &close);
  if (close) {  // the whole wave
    double wide[V], wkey[V], wgkey[V], total = 0.0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      wide[i] = p.sigmoid ? 1.0 / (1.0 + exp(-(double)v[i])) : exp((double)v[i] - (double)m);
      total += wide[i];
    }
    if (!p.sigmoid) {
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) total += __shfl_xor(total, o, 64);
#pragma unroll
      for (int i = 0; i < V; ++i) wide[i] /= total;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const bool can = v[i] > -INFINITY;
      const double c = p.bias ? wide[i] + (double)bias[i] : wide[i];
      wkey[i] = !can ? -(double)INFINITY : p.bias ? c : (double)v[i];
      wgkey[i] = !can ? -(double)INFINITY : p.bias || sums ? c : (double)v[i];
    }
    e = choose<V, double>(p, wkey, wgkey, -1.0, -1.0, scr, &close);
  }
  float* held = (float*)scr;
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (V * lane + i < p.E) held[V * lane + i] = s[i];
  wave_sync();
  float w = e >= 0 ? held[e] : 0.f;
  wave_sync();
  float scale = p.scale;
  if (p.renorm) scale /= lanes_reduce<64, AddOp>(w) + kTiny;
  *weight = e < 0 ? 0.f : nan ? __builtin_nanf("") : w * scale;
  return e;
}

// Exclusive sum over threads 0..255 (each its own count; others 0); total in all threads.
__device__ __forceinline__ int scan256(int v, int* wave_sums, int* total) {
  const int t = threadIdx.x, lane = t & 63;
  int s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(s, o, 64);
    if (lane >= o) s += u;
  }
  if (t < 256 && lane == 63) wave_sums[t >> 6] = s;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int x = wave_sums[w];
    if (w < (t >> 6)) before += x;
    all += x;
  }
  *total = all;
  return before + s - v;
}

struct PlaceLds {
  uint32_t bits[MIRA_MAX_EXPERTS][kWords];
  int base[MIRA_MAX_EXPERTS];
  int wave_sums[4];
};

// Order and positions of a chunk's pairs, by the whole workgroup.  sel(i) is the expert
// of pair i of the chunk, kept(t) whether its token t has shared experts; total(g) the pairs
// of group g in the call, before(g) those in earlier chunks.
template <typename Sel, typename Kept, typename Total, typename Before>
__device__ __forceinline__ void place_pairs(const SelectParams& p, PlaceLds& L, int chunk, Sel sel, Kept kept, Total total, Before before) {
  const int t = threadIdx.x, G = p.E + p.S, t0 = chunk * p.chunk, n = min(p.chunk, p.T - t0);
  for (int i = t; i < G * kWords; i += kThreads) (&L.bits[0][0])[i] = 0;
  int all;
  const int mine = t < G ? total(t) : 0;
  const int off = scan256(mine, L.wave_sums, &all);  // (its barrier: the bits are zero)
  if (t < G) {
    L.base[t] = off + before(t);
    if (chunk == 0) {
      if (p.counts_out) p.counts_out[t] = mine;
      if (p.offsets_out) p.offsets_out[t] = off;
    }
  }
  if (chunk == 0 && t == 0 && p.offsets_out) p.offsets_out[G] = all;
  const int routed = n * p.k, pairs = routed + n * p.S;
  auto pair_of = [&](int i, int* tok) {  // the group of pair i of the chunk, or -1
    if (i < routed) {
      *tok = i / p.k;
      return sel(i);
    }
    const int s = (i - routed) / n;
    *tok = i - routed - s * n;
    return kept(*tok) ? p.E + s : -1;
  };
  for (int i = t; i < pairs; i += kThreads) {
    int tok;
    const int g = pair_of(i, &tok);
    if (g >= 0) atomicOr(&L.bits[g][tok >> 5], 1u << (tok & 31));
  }
  __syncthreads();
  const size_t P = (size_t)p.T * (p.k + p.S), Tk = (size_t)p.T * p.k;
  for (int i = t; i < pairs; i += kThreads) {
    int tok;
    const int g = pair_of(i, &tok);
    const size_t pair = i < routed ? (size_t)t0 * p.k + i : Tk + (size_t)((i - routed) / n) * p.T + t0 + tok;
    int at = -1;
    if (g >= 0) {
      at = L.base[g] + __popc(L.bits[g][tok >> 5] & ((1u << (tok & 31)) - 1u));
      for (int w = 0; w < (tok >> 5); ++w) at += __popc(L.bits[g][w]);
      if (p.order) p.order[at] = (int)pair;
    }
    if (p.pos) p.pos[pair] = at;
  }
  if (p.order)
    for (size_t i = (size_t)all + (size_t)chunk * kThreads + t; i < P; i += (size_t)p.chunks * kThreads) p.order[i] = -1;
}

// A chunk of tokens: a wave takes a row at a time.  One chunk places its pairs at once
// (ONE); several leave their counts.
template <int V, bool ONE, typename T>
__global__ __launch_bounds__(kThreads) void route_select_kernel(SelectParams p) {
  __shared__ double scr[kWaves][MIRA_MAX_EXPERTS];
  __shared__ int hist[MIRA_MAX_EXPERTS];
  __shared__ int kept;
  __shared__ int16_t sel[ONE ? kChunk * MIRA_MAX_TOPK : 1];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int t0 = blockIdx.x * p.chunk, n = min(p.chunk, p.T - t0);
  if (t < MIRA_MAX_EXPERTS) hist[t] = 0;
  if (t == 0) kept = 0;
  float bias[V], bias_max = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    bias[i] = p.bias && V * lane + i < p.E ? p.bias[V * lane + i] : 0.f;
    bias_max = fmaxf(bias_max, fabsf(bias[i]));
  }
  bias_max = lanes_reduce<64, MaxOp>(bias_max);
  __syncthreads();
  for (int i = wave; i < n; i += kWaves) {
    float w;
    const int e = select_row<V, T>(p, t0 + i, bias, bias_max, scr[wave], &w);
    if (lane < p.k) {
      const size_t at = (size_t)(t0 + i) * p.k + lane;
      p.idx[at] = e;
      if (p.weight) p.weight[at] = w;
      if (p.place) {
        if (ONE) sel[i * p.k + lane] = (int16_t)e;
        if (e >= 0) atomicAdd(&hist[e], 1);
      }
    }
    if (p.place && lane == 0 && (!p.mask || p.mask[t0 + i])) atomicAdd(&kept, 1);
  }
  if (!p.place) return;
  __syncthreads();
  auto count = [&](int g) { return g < p.E ? hist[g] : kept; };
  if constexpr (ONE) {
    __shared__ PlaceLds place;
    place_pairs(p, place, 0, [&](int i) { return (int)sel[i]; }, [&](int i) { return !p.mask || p.mask[i] != 0; }, count,
                [](int) { return 0; });
  } else {
    if (t < p.E + p.S) p.counts[(size_t)blockIdx.x * (p.E + p.S) + t] = count(t);
  }
}

// For each group the chunks' counts to sums of those before, and the total.
__global__ __launch_bounds__(256) void route_scan_kernel(SelectParams p) {
  __shared__ int wave_sums[2][4];
  const int G = p.E + p.S, g = blockIdx.x;
  int run = 0, turn = 0;
  for (int c0 = 0; c0 < p.chunks; c0 += 256, turn ^= 1) {
    const int c = c0 + threadIdx.x;
    int* at = p.counts + (size_t)c * G + g;
    const int v = c < p.chunks ? *at : 0;
    int all;
    const int before = scan256(v, wave_sums[turn], &all);
    if (c < p.chunks) *at = run + before;
    run += all;
  }
  if (threadIdx.x == 0) p.totals[g] = run;
}

__global__ __launch_bounds__(kThreads) void route_place_kernel(SelectParams p) {
  __shared__ PlaceLds place;
  const int chunk = blockIdx.x, t0 = chunk * p.chunk;
  const int32_t* idx = p.idx + (size_t)t0 * p.k;
  place_pairs(p, place, chunk, [&](int i) { return (int)idx[i]; }, [&](int i) { return !p.mask || p.mask[t0 + i] != 0; },
              [&](int g) { return p.totals[g]; }, [&](int g) { return p.counts[(size_t)chunk * (p.E + p.S) + g]; });
}

// Tokens of a chunk: 32 until the chunks fill the CUs, then more, in steps of 32.
int chunk_tokens(int T) {
  const int c = ((T + 255) / 256 + 31) / 32 * 32;
  return c < 32 ? 32 : c > kChunk ? kChunk : c;
}
int chunk_count(int T) { return (int)(((int64_t)T + chunk_tokens(T) - 1) / chunk_tokens(T)); }

template <int V, typename T>
void launch_select(const SelectParams& p, hipStream_t st) {
  if (p.chunks == 1)
    launch_timed("route_select", route_select_kernel<V, true, T>, dim3(1), dim3(kThreads), 0, st, p);
  else
    launch_timed("route_select", route_select_kernel<V, false, T>, dim3(p.chunks), dim3(kThreads), 0, st, p);
}

template <typename T>
void launch_select_of(const SelectParams& p, hipStream_t st) {
  if (p.E <= 64) launch_select<1, T>(p, st);
  else if (p.E <= 128) launch_select<2, T>(p, st);
  else launch_select<4, T>(p, st);
}

// ---- the weights' gradient ----------------------------------------------------

struct SelectGradParams {
  const void* logits;
  const int32_t* idx;
  const float* dweight;
  const void* add;  // may be null
  void* d;
  size_t ld, ld_add, ld_d;
  int T, E, k;
  bool sigmoid, renorm;
  float scale;
};

__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(uint16_t* p, float v) { *p = __builtin_bit_cast(uint16_t, (__bf16)v); }

// A row to L lanes, four experts l, l + L, .. to a lane; k <= L lanes hold its selection.
//   ds_e = scale (g_e - [renorm] A / D) / D on the selected, A = sum g s, D = sum s + 1e-20 (1 without renorm);
//   sigmoid: dl_e = ds_e s_e (1 - s_e);  softmax: dl_e = s_e (ds_e - B), B = sum ds s, which with
//   renorm is scale (A / D) (1e-20 / D): as a difference of its terms nothing of it would be left.
template <int L, typename T>
__global__ __launch_bounds__(256) void route_select_grad_kernel(SelectGradParams p) {
  const int l = threadIdx.x % L;
  // (whole groups of lanes leave the loop)
  for (size_t row = (size_t)blockIdx.x * (256 / L) + threadIdx.x / L; row < (size_t)p.T; row += (size_t)gridDim.x * (256 / L)) {
    int sel = -1;
    float g = 0.f;
    if (l < p.k) {
      sel = p.idx[row * p.k + l];
      if ((uint32_t)sel >= (uint32_t)p.E) sel = -1;
      if (sel >= 0) g = p.dweight[row * p.k + l];
    }
    const T* x = (const T*)p.logits + row * p.ld;
    float v[4], ge[4] = {0.f, 0.f, 0.f, 0.f}, n[4] = {0.f, 0.f, 0.f, 0.f};
  #pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = l + L * i < p.E ? load_act(x, l + L * i) : -INFINITY;
    bool any = false;
    for (int j = 0; j < p.k; ++j) {
      const int e = __shfl(sel, j, L);
      const float ge_j = __shfl(g, j, L);
      any |= e >= 0;
  #pragma unroll
      for (int i = 0; i < 4; ++i)
        if (e == l + L * i) {
          ge[i] += ge_j;
          n[i] += 1.f;
        }
    }
    float s[4], rest[4];  // scores, and 1 - s for sigmoid
    if (p.sigmoid) {
  #pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e = exp_neg(-fabsf(v[i])), r = __builtin_amdgcn_rcpf(1.f + e);
        const bool up = v[i] >= 0.f;
        s[i] = n[i] > 0.f ? (up ? r : e * r) : 0.f;
        rest[i] = up ? e * r : r;
      }
    } else {
      float m = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
      m = lanes_reduce<L, MaxOp>(m);
      m = m == -INFINITY ? 0.f : m;
      float sum = 0.f;
  #pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[i] = exp_neg(v[i] - m);
        sum += s[i];
      }
      sum = lanes_reduce<L, AddOp>(sum);
      const float inv = sum == 0.f ? 0.f : __builtin_amdgcn_rcpf(sum);
  #pragma unroll
      for (int i = 0; i < 4; ++i) s[i] *= inv;
    }
    float A = 0.f, D = 0.f;
  #pragma unroll
    for (int i = 0; i < 4; ++i) {
      A = fmaf(ge[i], s[i], A);
      D = fmaf(n[i], s[i], D);
    }
    A = lanes_reduce<L, AddOp>(A);
    D = lanes_reduce<L, AddOp>(D) + kTiny;
    const float inv = p.renorm ? 1.f / D : 1.f, mean = p.renorm ? A * inv : 0.f;
    const float B = p.scale * (p.renorm ? mean * (kTiny * inv) : A);
    T* d = (T*)p.d + row * p.ld_d;
  #pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = l + L * i;
      if (e >= p.E) continue;
      const float ds = p.scale * inv * (ge[i] - n[i] * mean);
      float o = !any ? 0.f : p.sigmoid ? ds * s[i] * rest[i] : s[i] * (ds - B);
      if (p.sigmoid && n[i] == 0.f) o = 0.f;
      if (p.add) o += load_act((const T*)p.add + row * p.ld_add, e);
      store1(d + e, o);
    }
  }
}

__global__ void pairs_fill_kernel(int32_t* pos, int n) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < (size_t)n; i += (size_t)gridDim.x * 256) pos[i] = -1;
}
__global__ void pairs_invert_kernel(const int32_t* order, int m, int n, int32_t* pos) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < (size_t)m; i += (size_t)gridDim.x * 256) {
    const int p = order[i];
    if (p >= 0 && p < n) pos[p] = (int32_t)i;
  }
}

uint32_t grid_of(int n) { return ((uint32_t)n + 255) / 256; }

}  // namespace

size_t route_select_ws_bytes(int T, int E, int S) {
  const size_t G = (size_t)E + S;
  // the most chunks that any call of up to T tokens has: chunks of 32 up to 8192 tokens, 256 chunks up to 65536
  const size_t chunks = T <= 8192 ? ((size_t)T + 31) / 32 : T <= 65536 ? 256 : ((size_t)T + kChunk - 1) / kChunk;
  return align_up((chunks < 1 ? 1 : chunks) * G * 4, 256) + align_up(G * 4, 256);
}

hipError_t launch_route_select(const mira_route_select_args& a, hipStream_t st) {
  SelectParams p{};
  p.logits = a.logits;
  p.bias = a.bias;
  p.mask = a.mask;
  p.idx = a.topk_idx;
  p.weight = a.topk_weight;
  p.counts_out = a.expert_counts;
  p.offsets_out = a.expert_offsets;
  p.order = a.pair_order;
  p.pos = a.pair_pos;
  p.ld = a.ld_logits ? a.ld_logits : a.n_experts;
  p.T = a.n_tokens;
  p.E = a.n_experts;
  p.k = a.top_k;
  p.S = a.n_shared;
  p.groups = a.top_groups == a.n_groups ? 1 : a.n_groups;  // all groups kept is none
  p.top_groups = a.top_groups;
  p.best = a.group_best;
  p.chunk = chunk_tokens(p.T);
  p.chunks = chunk_count(p.T < 1 ? 1 : p.T);
  p.sigmoid = a.flags & MIRA_ROUTE_SIGMOID;
  p.renorm = a.flags & MIRA_ROUTE_RENORM;
  p.scale = a.scale;
  p.place = p.counts_out || p.offsets_out || p.order || p.pos;
  const int G = p.E + p.S;
  p.counts = (int32_t*)a.workspace;
  p.totals = (int32_t*)((char*)a.workspace + align_up((size_t)p.chunks * G * 4, 256));
  if (a.logits_dtype == MIRA_F32) launch_select_of<float>(p, st);
  else launch_select_of<uint16_t>(p, st);
  if (p.place && p.chunks > 1) {
    launch_timed("route_scan", route_scan_kernel, dim3(G), dim3(256), 0, st, p);
    launch_timed("route_place", route_place_kernel, dim3(p.chunks), dim3(kThreads), 0, st, p);
  }
  return hipGetLastError();
}

hipError_t launch_route_select_grad(const mira_route_select_grad_args& a, hipStream_t st) {
  SelectGradParams p{};
  p.logits = a.logits;
  p.idx = a.topk_idx;
  p.dweight = a.dweight;
  p.add = a.add;
  p.d = a.dlogits;
  p.ld = a.ld_logits ? a.ld_logits : a.n_experts;
  p.ld_add = a.ld_add ? a.ld_add : a.n_experts;
  p.ld_d = a.ld_dlogits ? a.ld_dlogits : a.n_experts;
  p.T = a.n_tokens;
  p.E = a.n_experts;
  p.k = a.top_k;
  p.sigmoid = a.flags & MIRA_ROUTE_SIGMOID;
  p.renorm = a.flags & MIRA_ROUTE_RENORM;
  p.scale = a.scale;
  const bool f32 = a.logits_dtype == MIRA_F32;
  if (p.E <= 64) {
    const dim3 grid(min((p.T + 15) / 16, kMaxGrid));
    launch_timed("route_select_grad", f32 ? route_select_grad_kernel<16, float> : route_select_grad_kernel<16, uint16_t>, grid, dim3(256), 0, st, p);
  } else {
    const dim3 grid(min((p.T + 3) / 4, kMaxGrid));
    launch_timed("route_select_grad", f32 ? route_select_grad_kernel<64, float> : route_select_grad_kernel<64, uint16_t>, grid, dim3(256), 0, st, p);
  }
  return hipGetLastError();
}

hipError_t launch_pair_positions(const int32_t* order, int m, int n_pairs, int32_t* pos, hipStream_t st) {
  if (n_pairs > 0) launch_timed("pair_fill", pairs_fill_kernel, dim3(grid_of(n_pairs)), dim3(256), 0, st, pos, n_pairs);
  if (m > 0) launch_timed("pair_positions", pairs_invert_kernel, dim3(grid_of(m)), dim3(256), 0, st, order, m, n_pairs, pos);
  return hipGetLastError();
}

}  // namespace mira
