// Balance loss of a router, its per-expert counts and its gradient.
//
//   loss_g = coef * sum_e f_ge P_ge,  f_ge = E c_ge / (k n_g),  P_ge = mean of p_te,
//   d/dlogit_te = grad_g * (coef / n_g) * p_te * (f_ge - sum_j f_gj p_tj),
// with c the counts of the selected experts and p the row softmax.  The
// gradient needs the counts of the whole group but not P, so the counts (which
// read the small topk_idx only) come first and one pass over the logits then
// gives both the gradient and the sums of p: the logits are read once and the
// gradient written once.
//
// A long call is bound by memory: 131072 rows of 256 in fp32 with their gradient,
// 273 MB, 72 us, of which the pass over the logits takes 57 to 63 at 4.3 to 4.7 TB/s (a copy
// runs at 5.1).  A short one is bound by its launches and by loads that wait for one
// another: 16 rows of 8 5.9 us, 2048 of 64 12 us.  Where a comment compares two ways,
// both were timed with the rest of the file as it was then; calls may be faster now.
//
// Rows are split into at most kMaxChunks chunks, a workgroup each; a chunk
// walks the groups that it meets.  Over the chunks in order, (chunk, group)
// pairs that meet only ever step one of the two up, so chunk + group numbers
// the partial sums without gaps to search: kMaxChunks + G slots hold any
// layout of groups.  A group's slots are added in order to its means and loss: for
// one group by the last chunk to end, for several in a launch that follows (37
// groups of 30011 rows: 26 us so, 24 today, and 32 with the chunks counting their
// groups' ends; one group of 2048 x 64: 17 us with the launch, 12 without).  Calls of
// few logits run one workgroup per group in a single launch.
#include "device_util.h"
#include "mira_internal.h"

namespace mira {

namespace {

constexpr int kMaxChunks = 256;   // one 1024-thread workgroup per CU
constexpr int kBigThreads = 1024;
// Selections that one workgroup per group counts; more are counted by chunks, after
// a launch that zeroes the counts (us, per group against chunks: one group of 32768
// 15.9 and 17.1, of 49152 17.8 and 17.3; 37 groups of 3244 26.5 and 29.3, 16 of 8192
// 31.5 and 27.9, 4 of 65536 31 and 22).  Beyond 2^18 of them one group may hold so
// many that its workgroup is what the call waits for: 40 to 90 us at 2^18.
constexpr bool few_pairs(size_t pairs, size_t groups) {
  return pairs <= 32768 || (pairs <= groups * 4096 && pairs <= 1u << 18);
}

struct BalanceParams {
  const void* logits;
  const int32_t* idx;
  const int32_t* offsets;  // may be null
  const uint8_t* mask;     // may be null
  const float* grad_loss;  // may be null
  void* dlogits;           // may be null
  int32_t* counts;         // output or workspace
  int32_t* kept;           // [G] rows kept (with a mask)
  int32_t* ended;          // chunks that have ended (one group)
  float* mean;             // may be null
  float* loss;             // may be null
  float* partial;          // [chunks + G][E]
  size_t ld_x, ld_d;
  int T, E, k, G, chunk_rows;
  float coef;
  uint64_t inv_k;  // 2^34 / k rounded up: i / k = i * inv_k >> 34 for i < 2^30, k <= 16
};

// The logits of a row that a lane holds, up to four: VEC: 4l .. 4l+3 (E a multiple
// of 4, rows aligned to four elements), else l, l+L, l+2L, l+3L.  FEW: the largest power
// of two of lanes that the experts fill, at most two values a lane; four would leave
// most lanes of so short a row without any.
constexpr int kFewExperts = 8;
template <int L, bool VEC>
__device__ __forceinline__ int expert_of(int l, int i) {
  return VEC ? 4 * l + i : l + L * i;
}
template <int L, bool VEC, typename T>
__device__ __forceinline__ void load_row(const T* row, int l, int E, float v[4]) {
  if constexpr (VEC) {
    if (4 * l < E) {
      load4_act(row + 4 * l, v);
    } else {
      v[0] = v[1] = v[2] = v[3] = -INFINITY;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = l + L * i;
      v[i] = e < E ? load_act(row, e) : -INFINITY;
    }
  }
}
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
// (a NaN keeps its upper half: the rounding increment must not carry it into infinity or zero)
__device__ __forceinline__ uint16_t to_bf16(float v) {
  return v != v ? (uint16_t)((__float_as_uint(v) >> 16) | 0x40u) : f32_to_bf16_rne(v);
}
__device__ __forceinline__ void store1(uint16_t* p, float v) { *p = to_bf16(v); }
__device__ __forceinline__ void store4(float* p, const float v[4]) { *(v4f*)p = v4f{v[0], v[1], v[2], v[3]}; }
__device__ __forceinline__ void store4(uint16_t* p, const float v[4]) {
  *(uint2*)p = uint2{(uint32_t)to_bf16(v[0]) | (uint32_t)to_bf16(v[1]) << 16,
                     (uint32_t)to_bf16(v[2]) | (uint32_t)to_bf16(v[3]) << 16};
}
template <int L, bool VEC, typename T>
__device__ __forceinline__ void store_row(T* row, int l, int E, const float v[4]) {
  if constexpr (VEC) {
    if (4 * l < E) store4(row + 4 * l, v);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = l + L * i;
      if (e < E) store1(row + e, v[i]);
    }
  }
}

// Group bounds, clamped so that any offsets stay inside the buffers.
struct Segment {
  int lo, hi;
};
__device__ __forceinline__ Segment group_rows(const BalanceParams& q, int g) {
  if (!q.offsets) return Segment{0, q.T};
  const int lo = min(max(q.offsets[g], 0), q.T);
  return Segment{lo, min(max(q.offsets[g + 1], lo), q.T)};
}
__device__ __forceinline__ float count_scale(const BalanceParams& q, int n) {
  return n > 0 ? (float)q.E * (1.f / ((float)q.k * (float)n)) : 0.f;
}
__device__ __forceinline__ float group_grad(const BalanceParams& q, int g) { return q.grad_loss ? q.grad_loss[g] : 1.f; }
__device__ __forceinline__ float grad_scale(const BalanceParams& q, float grad, int n) {
  return n > 0 ? grad * q.coef / (float)n : 0.f;
}

// Softmax, gradient and sums of p of rows lo, lo + step, .. < hi for one lane
// group of L lanes (lane l of it); acc holds the lane's sums of p.  U rows are
// in flight at once.
// STEP (few experts, all of them selected): expf and the formula's own operations,
// each rounded once and none contracted.  The gradient is zero then but for its
// roundings, and these are those of the formula evaluated step by step, not of a
// rearrangement.  Either way they are fewer than 24 half steps; that costs little where
// rows are short (131072 of 8: 21.9 us, 20.7 without) and more from 9 experts on (of
// 16: 25.1 against 20.6, 500 of 16: 9.4 against 5.7), which therefore never take it.
template <int L, bool VEC, bool FEW, bool STEP, int U, typename T>
__device__ __forceinline__ void rows_pass(const BalanceParams& q, int lo, int hi, int step, int l,
                                          const int counts[4], int n, float grad, float acc[4]) {
  static_assert(FEW || !STEP, "few experts");
  constexpr int NV = FEW ? 2 : 4;  // values that a lane may hold
  const bool two = !FEW || q.E > L;  // the lanes' second values exist (FEW: E is no power of two)
  const T* x = (const T*)q.logits;
  T* d = (T*)q.dlogits;
  for (int r0 = lo; r0 < hi; r0 += U * step) {
    float v[U][4];
    bool keep[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * step;
      keep[u] = r < hi;
      if (r < hi) {
        load_row<L, VEC>(x + (size_t)r * q.ld_x, l, q.E, v[u]);
        if (q.mask) keep[u] = q.mask[r] != 0;
      }
    }
    // (here, so that the first rows do not wait for the counts to arrive)
    const float gscale = grad_scale(q, grad, n), cs = count_scale(q, n);
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = (float)counts[i] * cs;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * step;
      if (r >= hi) break;
      float m = v[u][0];
#pragma unroll
      for (int i = 1; i < NV; ++i) m = fmaxf(m, v[u][i]);
      m = lanes_reduce<L, MaxOp>(m);
      m = m == -INFINITY ? 0.f : m;
      float o[4] = {0.f, 0.f, 0.f, 0.f};
      if constexpr (STEP) {
#pragma clang fp contract(off)
        float e0 = expf(v[u][0] - m), e1 = two ? expf(v[u][1] - m) : 0.f;
        const float s = lanes_reduce<L, AddOp>(e0 + e1);
        e0 = s == 0.f ? 0.f : e0 / s;
        if (two) e1 = s == 0.f ? 0.f : e1 / s;
        const float f0 = f[0] * e0, f1 = f[1] * e1;
        const float w = lanes_reduce<L, AddOp>(f0 + f1);
        acc[0] += keep[u] ? e0 : 0.f;
        o[0] = keep[u] ? (gscale * e0) * (f[0] - w) : 0.f;
        if (two) {
          acc[1] += keep[u] ? e1 : 0.f;
          o[1] = keep[u] ? (gscale * e1) * (f[1] - w) : 0.f;
        }
      } else {
        float s = 0.f, w = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if (i == 1 && !two) break;
          v[u][i] = exp_neg(v[u][i] - m);
          s += v[u][i];
          w = fmaf(f[i], v[u][i], w);
        }
        s = lanes_reduce<L, AddOp>(s);
        w = lanes_reduce<L, AddOp>(w);
        const float inv = s == 0.f ? 0.f : __builtin_amdgcn_rcpf(s);
        w *= inv;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if (i == 1 && !two) break;
          const float p = v[u][i] * inv;
          acc[i] += keep[u] ? p : 0.f;
          o[i] = keep[u] ? gscale * p * (f[i] - w) : 0.f;
        }
      }
      if (d) store_row<L, VEC>(d + (size_t)r * q.ld_d, l, q.E, o);
    }
  }
}

// Sum over the lane groups of the workgroup: sums[e] for e < E, in LDS.
template <int L, bool VEC, int THREADS>
__device__ __forceinline__ void reduce_groups(float acc[4], int E, float (*wave_sums)[MIRA_MAX_EXPERTS]) {
  const int lane = threadIdx.x & 63, l = lane % L, wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int o = L; o < 64; o <<= 1) acc[i] += __shfl_xor(acc[i], o, 64);
    const int e = expert_of<L, VEC>(l, i);
    if (lane < L && e < E) wave_sums[wave][e] = acc[i];
  }
}

// Counts the pairs of rows [lo, hi) into hist and the kept rows into *kept
// (both in LDS, zeroed before).  Four loads of each thread are in flight, and a
// pair's row comes by a product instead of a division (3904 masked rows of 5 of 5
// experts: 24 us the call without, 17 so).  Counters of few experts are met by many
// lanes at once; counts in registers, added up by the waves, were not faster (1024
// rows of 2 of 8: 9.2 us so, 10.4 in registers).
template <int THREADS>
__device__ __forceinline__ void count_pairs(const BalanceParams& q, int lo, int hi, int* hist, int* kept) {
  const uint32_t end = (uint32_t)hi * q.k;  // T * k is at most 2^30
  constexpr int kFlight = 4;
  for (uint32_t i = (uint32_t)lo * q.k + threadIdx.x; i < end; i += kFlight * THREADS) {
    int e[kFlight], keep[kFlight];
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      e[j] = q.idx[min(i + j * THREADS, end - 1)];
      keep[j] = 1;
    }
    if (q.mask) {  // (no load behind a condition of its own: it would be waited for before the next)
#pragma unroll
      for (int j = 0; j < kFlight; ++j)
        keep[j] = q.mask[(uint32_t)((uint64_t)min(i + j * THREADS, end - 1) * q.inv_k >> 34)];
    }
#pragma unroll
    for (int j = 0; j < kFlight; ++j)
      if (i + j * THREADS < end && keep[j] && (uint32_t)e[j] < (uint32_t)q.E) atomicAdd(hist + e[j], 1);
  }
  if (q.mask) {
    int n = 0;
    for (int r = lo + threadIdx.x; r < hi; r += THREADS) n += q.mask[r] != 0;
    if (n) atomicAdd(kept, n);
  }
}

// One workgroup per group: counts, rows, means and loss.  Bound by latency: a launch,
// the counts' loads, then the rows' (16 rows of 8 experts 3.1 us of the call's 5.9).
template <int L, bool VEC, bool FEW, bool STEP, int THREADS, typename T>
__global__ __launch_bounds__(THREADS) void balance_group_kernel(BalanceParams q) {
  __shared__ int hist[MIRA_MAX_EXPERTS];
  __shared__ int kept;
  __shared__ float wave_sums[THREADS / 64][MIRA_MAX_EXPERTS];
  __shared__ float part[THREADS / 64];
  const int g = blockIdx.x, t = threadIdx.x, l = t % L;
  const Segment s = group_rows(q, g);
  for (int e = t; e < q.E; e += THREADS) hist[e] = 0;
  if (t == 0) kept = 0;
  __syncthreads();
  count_pairs<THREADS>(q, s.lo, s.hi, hist, &kept);
  __syncthreads();
  const int n = q.mask ? kept : s.hi - s.lo;
  const float cs = count_scale(q, n);
  int counts[4];
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = expert_of<L, VEC>(l, i);
    counts[i] = e < q.E ? hist[e] : 0;
  }
  rows_pass<L, VEC, FEW, STEP, FEW ? 4 : 2, T>(q, s.lo + t / L, s.hi, THREADS / L, l, counts, n, group_grad(q, g), acc);
  reduce_groups<L, VEC, THREADS>(acc, q.E, wave_sums);
  __syncthreads();
  float term = 0.f;
  for (int e = t; e < q.E; e += THREADS) {
    float sum = 0.f;
    for (int w = 0; w < THREADS / 64; ++w) sum += wave_sums[w][e];
    const float mean = n > 0 ? sum / (float)n : 0.f;
    if (q.mean) q.mean[(size_t)g * q.E + e] = mean;
    q.counts[(size_t)g * q.E + e] = hist[e];
    term += (float)hist[e] * cs * mean;
  }
  term = wave_sum(term);
  if ((t & 63) == 0) part[t >> 6] = term;
  __syncthreads();
  if (t == 0 && q.loss) {
    float sum = 0.f;
    for (int w = 0; w < THREADS / 64; ++w) sum += part[w];
    q.loss[g] = q.coef * sum;
  }
}

// ---- many logits ----------------------------------------------------------------

__global__ __launch_bounds__(256) void balance_zero_kernel(int32_t* counts, size_t n, int32_t* kept, int32_t* ended, int G) {
  if (blockIdx.x == 0 && threadIdx.x == 0) *ended = 0;
  const size_t i0 = (size_t)blockIdx.x * 256 + threadIdx.x, step = (size_t)gridDim.x * 256;
  for (size_t i = i0; i < n; i += step) counts[i] = 0;
  for (size_t i = i0; i < (size_t)G; i += step) kept[i] = 0;
}

// Few pairs: one workgroup per group counts them, no zeros and no second pass.
__global__ __launch_bounds__(kBigThreads) void balance_count_group_kernel(BalanceParams q) {
  __shared__ int hist[MIRA_MAX_EXPERTS];
  __shared__ int kept;
  const int g = blockIdx.x;
  const Segment s = group_rows(q, g);
  for (int e = threadIdx.x; e < q.E; e += kBigThreads) hist[e] = 0;
  if (threadIdx.x == 0) kept = 0;
  __syncthreads();
  count_pairs<kBigThreads>(q, s.lo, s.hi, hist, &kept);
  __syncthreads();
  for (int e = threadIdx.x; e < q.E; e += kBigThreads) q.counts[(size_t)g * q.E + e] = hist[e];
  if (threadIdx.x == 0) {
    q.kept[g] = kept;
    if (g == 0) *q.ended = 0;
  }
}

// Walks the groups that rows [lo, hi) meet, upwards: f(g, the group's rows, first
// row, end row).  The whole workgroup looks at all offsets at once for the group
// that holds a row; a search would wait for memory at every step.
template <typename F>
__device__ __forceinline__ void for_groups(const BalanceParams& q, int lo, int hi, F&& f) {
  if (!q.offsets) {
    if (lo < hi) f(0, Segment{0, q.T}, lo, hi);
    return;
  }
  __shared__ int found[3];
  int row = lo, above = -1, g = -1;
  Segment s{0, 0};
  while (true) {
    if (g >= 0 && g + 1 < q.G) s = group_rows(q, g + 1);  // mostly the next one
    if (g >= 0 && g + 1 < q.G && s.lo <= row && row < s.hi) {
      ++g;
    } else {
      __syncthreads();
      if (threadIdx.x == 0) found[0] = -1;
      __syncthreads();
      row = max(row, min(max(q.offsets[0], 0), q.T));
      for (int i = threadIdx.x; i < q.G; i += blockDim.x) {
        const Segment at = group_rows(q, i);
        if (at.lo <= row && row < at.hi) {  // one group, where the offsets ascend
          found[0] = i;
          found[1] = at.lo;
          found[2] = at.hi;
        }
      }
      __syncthreads();
      g = found[0];
      s = Segment{found[1], found[2]};
      // (none: past the last group; not above the last one: offsets that do not ascend)
      if (row >= hi || g <= above || s.lo > row || s.hi <= row) return;
    }
    f(g, s, row, min(s.hi, hi));
    above = g;
    row = s.hi;
    if (row >= hi) return;
  }
}

// Means and loss of a group from its chunks' sums: thread (e, part) adds every
// parts-th slot in order, then the parts are added in order.  The sums come from
// workgroups on other XCDs: both sides use agent-scope accesses, which pass the
// XCDs' own L2, and the writers wait for theirs to arrive before they count their
// chunk as ended.  (Agent-scope fences instead write all of an L2 back, the
// gradient's lines with it: 131072 x 256 took 137 us so, 75 us like this.)
__device__ __forceinline__ void finish_group(const BalanceParams& q, int g, const Segment& s, int n, float* sums) {
  int width = 1;
  while (width < q.E) width *= 2;
  const int t = threadIdx.x, e = t % width, part = t / width, parts = kBigThreads / width;
  float sum = 0.f;
  if (e < q.E && s.lo < s.hi) {
    const int c0 = s.lo / q.chunk_rows, c1 = (s.hi - 1) / q.chunk_rows;
    for (int c = c0 + part; c <= c1; c += 32 * parts) {  // 32 loads in flight, added in order
      float v[32];
#pragma unroll
      for (int i = 0; i < 32; ++i)
        v[i] = __hip_atomic_load(q.partial + (size_t)(min(c + i * parts, c1) + g) * q.E + e, __ATOMIC_RELAXED,
                                 __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
      for (int i = 0; i < 32; ++i) sum += c + i * parts <= c1 ? v[i] : 0.f;
    }
  }
  __syncthreads();
  sums[t] = sum;
  __syncthreads();
  float term = 0.f;
  if (part == 0 && e < q.E) {
    for (int i = 1; i < parts; ++i) sum += sums[i * width + e];
    const float mean = n > 0 ? sum / (float)n : 0.f;
    if (q.mean) q.mean[(size_t)g * q.E + e] = mean;
    term = (float)q.counts[(size_t)g * q.E + e] * count_scale(q, n) * mean;
  }
  __syncthreads();
  term = wave_sum(term);
  if ((t & 63) == 0) sums[t >> 6] = term;
  __syncthreads();
  if (t == 0 && q.loss) {
    float total = 0.f;
    for (int w = 0; w < kBigThreads / 64; ++w) total += sums[w];
    q.loss[g] = q.coef * total;
  }
}

// The one pass over the logits: a chunk of rows each workgroup, L lanes a row.  Bound
// by memory (131072 x 256 fp32: 57 to 63 us, 268 MB at 4.3 to 4.7 TB/s); 1024 threads on each CU and
// two rows of each lane group in flight measured best (512 threads and 512 chunks 86 us
// the call against 76 then; a scalar path for row lengths that are no multiple of four
// takes 76 where vectors at any alignment took 80).
template <int L, bool VEC, bool FEW, bool STEP, typename T>
__global__ __launch_bounds__(kBigThreads) void balance_rows_kernel(BalanceParams q) {
  __shared__ float wave_sums[kBigThreads / 64][MIRA_MAX_EXPERTS];
  __shared__ int last;
  const int t = threadIdx.x, l = t % L;
  const int lo = blockIdx.x * q.chunk_rows, hi = min(lo + q.chunk_rows, q.T);
  for_groups(q, lo, hi, [&](int g, Segment s, int a, int b) {
    int counts[4];
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    const int n = q.mask ? q.kept[g] : s.hi - s.lo;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = expert_of<L, VEC>(l, i);
      counts[i] = q.counts[(size_t)g * q.E + min(e, q.E - 1)];
    }
    rows_pass<L, VEC, FEW, STEP, FEW ? 4 : 2, T>(q, a + t / L, b, kBigThreads / L, l, counts, n, group_grad(q, g), acc);
    if (!q.mean && !q.loss) return;
    __syncthreads();
    reduce_groups<L, VEC, kBigThreads>(acc, q.E, wave_sums);
    __syncthreads();
    for (int e = t; e < q.E; e += kBigThreads) {
      float sum = 0.f;
      for (int w = 0; w < kBigThreads / 64; ++w) sum += wave_sums[w][e];
      __hip_atomic_store(q.partial + (size_t)(blockIdx.x + g) * q.E + e, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  });
  if (q.offsets || (!q.mean && !q.loss)) return;
  // One group: the last chunk to end finishes it.  (The sums have arrived when the
  // counter of stores in flight is zero.)
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (t == 0)
    last = __hip_atomic_fetch_add(q.ended, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
  __syncthreads();
  if (last) finish_group(q, 0, Segment{0, q.T}, q.mask ? q.kept[0] : q.T, &wave_sums[0][0]);
}

// Several groups: a workgroup each adds its chunks' sums (5 us: a launch and two
// loads that wait for one another).
__global__ __launch_bounds__(kBigThreads) void balance_finish_kernel(BalanceParams q) {
  __shared__ float sums[kBigThreads];
  const Segment s = group_rows(q, blockIdx.x);
  finish_group(q, blockIdx.x, s, q.mask ? q.kept[blockIdx.x] : s.hi - s.lo, sums);
}

// Many pairs: each chunk counts its rows' and adds them to zeroed counts (131072 x 8
// pairs, 4 MB: 7 us, and the launch that zeroes 1 to 5).
__global__ __launch_bounds__(kBigThreads) void balance_count_kernel(BalanceParams q) {
  __shared__ int hist[MIRA_MAX_EXPERTS];
  __shared__ int kept;
  const int lo = blockIdx.x * q.chunk_rows, hi = min(lo + q.chunk_rows, q.T);
  for_groups(q, lo, hi, [&](int g, Segment, int a, int b) {
    for (int e = threadIdx.x; e < q.E; e += kBigThreads) hist[e] = 0;
    if (threadIdx.x == 0) kept = 0;
    __syncthreads();
    count_pairs<kBigThreads>(q, a, b, hist, &kept);
    __syncthreads();
    // integers: the order of these additions does not change the result
    for (int e = threadIdx.x; e < q.E; e += kBigThreads)
      if (hist[e]) atomicAdd(q.counts + (size_t)g * q.E + e, hist[e]);
    if (threadIdx.x == 0 && kept) atomicAdd(q.kept + g, kept);
    __syncthreads();
  });
}

struct BalanceLayout {
  size_t counts, kept, ended, partial, total;
};
BalanceLayout balance_layout(int E, int G) {
  BalanceLayout w;
  w.counts = 0;
  w.kept = align_up((size_t)G * E * 4, 256);
  w.ended = w.kept + align_up((size_t)G * 4, 256);
  w.partial = w.ended + 256;
  w.total = w.partial + align_up((size_t)(kMaxChunks + G) * E * 4, 256);
  return w;
}

template <int L, bool VEC, bool FEW, bool STEP, typename T>
void launch_rows(const BalanceParams& q, bool small, int chunks, hipStream_t st) {
  // a group of more than one pass of 256 threads gets a larger workgroup
  if (small && (size_t)q.T * L <= (size_t)q.G * 256)
    launch_timed("balance_group", balance_group_kernel<L, VEC, FEW, STEP, 256, T>, dim3(q.G), dim3(256), 0, st, q);
  else if (small)
    launch_timed("balance_group", balance_group_kernel<L, VEC, FEW, STEP, kBigThreads, T>, dim3(q.G), dim3(kBigThreads), 0, st, q);
  else
    launch_timed("balance_rows", balance_rows_kernel<L, VEC, FEW, STEP, T>, dim3(chunks), dim3(kBigThreads), 0, st, q);
}

// Lanes of a row: the largest power of two up to E for few experts, else the
// smallest of four values a lane.
int row_lanes(int E) {
  int lanes = 1;
  if (E <= kFewExperts)
    while (lanes * 2 <= E) lanes *= 2;
  else
    while (lanes * 4 < E) lanes *= 2;
  return lanes;
}

template <bool STEP, typename T>
void launch_few(const BalanceParams& q, bool small, int chunks, hipStream_t st) {
  switch (row_lanes(q.E)) {
    case 1: return launch_rows<1, false, true, true, T>(q, small, chunks, st);  // (its expert is always selected)
    case 2: return launch_rows<2, false, true, STEP, T>(q, small, chunks, st);
    case 4: return launch_rows<4, false, true, STEP, T>(q, small, chunks, st);
    default: return launch_rows<8, false, true, STEP, T>(q, small, chunks, st);
  }
}
template <bool VEC, typename T>
void launch_many(const BalanceParams& q, bool small, int chunks, hipStream_t st) {
  switch (row_lanes(q.E)) {
    case 4: return launch_rows<4, VEC, false, false, T>(q, small, chunks, st);
    case 8: return launch_rows<8, VEC, false, false, T>(q, small, chunks, st);
    case 16: return launch_rows<16, VEC, false, false, T>(q, small, chunks, st);
    case 32: return launch_rows<32, VEC, false, false, T>(q, small, chunks, st);
    default: return launch_rows<64, VEC, false, false, T>(q, small, chunks, st);
  }
}
template <typename T>
void launch_typed(const BalanceParams& q, bool vec, bool small, int chunks, hipStream_t st) {
  if (q.E <= kFewExperts && q.k >= q.E) launch_few<true, T>(q, small, chunks, st);
  else if (q.E <= kFewExperts) launch_few<false, T>(q, small, chunks, st);
  else if (vec) launch_many<true, T>(q, small, chunks, st);
  else launch_many<false, T>(q, small, chunks, st);
}

}  // namespace

size_t balance_ws_bytes(int E, int G) { return balance_layout(E, G).total; }

hipError_t launch_balance(const mira_balance_args& a, hipStream_t st) {
  const BalanceLayout w = balance_layout(a.n_experts, a.n_groups);
  char* ws = (char*)a.workspace;
  BalanceParams q{};
  q.logits = a.logits;
  q.idx = a.topk_idx;
  q.offsets = a.offsets;
  q.mask = a.mask;
  q.grad_loss = a.grad_loss;
  q.dlogits = a.dlogits;
  q.counts = a.counts ? a.counts : (int32_t*)(ws + w.counts);
  q.kept = (int32_t*)(ws + w.kept);
  q.mean = a.mean_prob;
  q.loss = a.loss;
  q.ended = (int32_t*)(ws + w.ended);
  q.partial = (float*)(ws + w.partial);
  q.ld_x = a.ld_logits ? a.ld_logits : a.n_experts;
  q.ld_d = a.ld_dlogits ? a.ld_dlogits : a.n_experts;
  q.T = a.n_tokens;
  q.E = a.n_experts;
  q.k = a.top_k;
  q.G = a.n_groups;
  q.coef = a.coef;
  q.inv_k = ((1ull << 34) + a.top_k - 1) / a.top_k;
  const int lanes = row_lanes(q.E);
  const size_t esz = a.logits_dtype == MIRA_F32 ? 4 : 2;
  const bool vec = q.E % 4 == 0 && q.ld_x % 4 == 0 && (uintptr_t)q.logits % (4 * esz) == 0 &&
                   (!q.dlogits || (q.ld_d % 4 == 0 && (uintptr_t)q.dlogits % (4 * esz) == 0));
  // One workgroup per group: few logits, or many groups of few logits (1000 rows of
  // 256 experts in 500 groups: 6.5 us so, 37 by chunks that walk the groups; kept to
  // 2^20 logits, where one group of nearly all of them costs some 150 us).
  const size_t logits = (size_t)q.T * lanes * 4;  // as the lanes hold them
  const bool small = logits <= 32768 || (logits <= (size_t)q.G * 8192 && logits <= 1u << 20);
  int chunks = 0;
  if (!small) {
    // whole passes of the workgroup's lane groups, at most kMaxChunks chunks
    const int rows = kBigThreads / lanes;
    q.chunk_rows = (int)align_up((size_t)(q.T + kMaxChunks - 1) / kMaxChunks, rows);
    chunks = (q.T + q.chunk_rows - 1) / q.chunk_rows;
    if (few_pairs((size_t)q.T * q.k, q.G)) {
      launch_timed("balance_count", balance_count_group_kernel, dim3(q.G), dim3(kBigThreads), 0, st, q);
    } else {
      const size_t n = (size_t)q.G * q.E;
      const int zb = (int)((n + 255) / 256 < 1024 ? (n + 255) / 256 : 1024);
      launch_timed("balance_zero", balance_zero_kernel, dim3(zb), dim3(256), 0, st, q.counts, n, q.kept, q.ended, q.G);
      launch_timed("balance_count", balance_count_kernel, dim3(chunks), dim3(kBigThreads), 0, st, q);
    }
  }
  if (a.logits_dtype == MIRA_F32) launch_typed<float>(q, vec, small, chunks, st);
  else launch_typed<uint16_t>(q, vec, small, chunks, st);
  if (!small && q.offsets && (q.mean || q.loss))
    launch_timed("balance_finish", balance_finish_kernel, dim3(q.G), dim3(kBigThreads), 0, st, q);
  return hipGetLastError();
}

}  // namespace mira
