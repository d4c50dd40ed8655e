// Selection of experts from logits, the order of the (token, expert) pairs, and
// the gradient of the weights.
//
// Selection: 16 lanes take a row, V experts l, l + 16, .. to a lane.  A candidate is one
// 32-bit key: 24 bits of its c = s + bias in fixed point (without bias of its logit, whose
// order is that of s) and 255 - expert below, so that sorting and taking maxima move value and
// index at once and equal values give the lower expert.  A lane sorts its best four or five; k + 1
// times the row's largest head is taken.  What is cut off and what fp32 rounds may hide the
// order of two candidates: where two neighbours of the result, or the groups at the border,
// lie closer than that (see score_margin), or a lane's best do not suffice, or a logit is NaN, a
// whole wave does the row again with c in 64 bits.  In long batches of up to 64 experts a
// row is one or four lanes'.
//
// Order: a chunk of tokens is a workgroup.  Each expert has a bit for every token of the
// chunk, so a pair's rank in its expert's list is a count of bits: no order of atomics
// decides anything.  Counts of all chunks are added up by a launch in between.
//
// 131072 x 256 fp32, 8 selected of 4 of 8 groups, sigmoid and bias: 67 us (151 MB, for which a copy takes
// 29): 54 for the selection (some 610 instructions to four rows, in chains: the vector units are busy 57 % of
// the time at four waves a SIMD, a fifth of LDS cycles are conflicts), 5 for the counts, 9 for the order.
#include "fp8_dev.h"

namespace mira {

namespace {

constexpr int kThreads = 512;      // of a chunk's workgroup, kOneThreads where one chunk is all
constexpr int kOneThreads = 1024;
constexpr int kPlaceThreads = 1024;
constexpr int kChunk = 256;     // most tokens of a chunk
// Counts (chunks times groups) that every chunk's workgroup adds up for itself, instead of a launch
// in between (us with and without: 64 chunks of 66 groups 10.0 and 12.8, 256 of 66 12.9 and 13.8, 256
// of 256 21.3 and 20.3).
constexpr int kFewCounts = 32768;
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

// 1 / (1 + exp(-x)) without overflow, 4 steps.
__device__ __forceinline__ float sigmoid(float x) {
  const float e = exp_neg(-fabsf(x)), r = __builtin_amdgcn_rcpf(1.f + e);
  return x >= 0.f ? r : e * r;
}

// A wave's scratch: its four rows' candidates, or each lane's best two of eight groups, or
// c of one row in 64 bits with its groups' scores.
constexpr int kPairStride = 66;  // (lanes of eight groups read in different banks)
union SelectScratch {
  uint32_t part[4][MIRA_MAX_EXPERTS];
  uint2 pair[8][kPairStride];
  struct {
    double c[MIRA_MAX_EXPERTS];
    double group[MIRA_MAX_EXPERTS];
  } wide;
};

// Lane j < k of a row's (or the wave's) lanes: the j-th expert, or -1, and its weight.
struct Pick {
  int e;
  float w;
};

// The weights of a row's selection, held by 16 lanes: experts and their logits.
__device__ __forceinline__ Pick weigh(const SelectParams& p, int e, float v, float m, float inv_sum, bool nan) {
  const float s = e < 0 ? 0.f : p.sigmoid ? sigmoid(v) : exp_neg(v - m) * inv_sum;
  float scale = p.scale;
  if (p.renorm) scale *= __builtin_amdgcn_rcpf(lanes_reduce<16, AddOp>(s) + kTiny);
  return Pick{e, e < 0 ? 0.f : nan ? __builtin_nanf("") : s * scale};
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
__device__ __forceinline__ uint32_t max16_u(uint32_t v) {
  v = max(v, dpp_u<0xB1>(v));
  v = max(v, dpp_u<0x4E>(v));
  v = max(v, dpp_u<0x141>(v));
  return max(v, dpp_u<0x140>(v));
}
// Over the wave: of 64-bit values, and the least of 32-bit ones.
template <int CTRL>
__device__ __forceinline__ double dpp_d(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  return __longlong_as_double((long long)((uint64_t)dpp_u<CTRL>((uint32_t)(u >> 32)) << 32 | dpp_u<CTRL>((uint32_t)u)));
}
// (Both halves of 32 or 64 lanes swapped: one of the two results is the lane's own value.)
__device__ __forceinline__ double wave_max64(double v) {
  v = fmax(v, dpp_d<0xB1>(v));
  v = fmax(v, dpp_d<0x4E>(v));
  v = fmax(v, dpp_d<0x141>(v));
  v = fmax(v, dpp_d<0x140>(v));
  uint64_t u = (uint64_t)__double_as_longlong(v);
  auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)u, false, false);
  auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
  v = fmax(__longlong_as_double((long long)((uint64_t)hi[0] << 32 | lo[0])), __longlong_as_double((long long)((uint64_t)hi[1] << 32 | lo[1])));
  u = (uint64_t)__double_as_longlong(v);
  lo = __builtin_amdgcn_permlane32_swap((uint32_t)u, (uint32_t)u, false, false);
  hi = __builtin_amdgcn_permlane32_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
  return fmax(__longlong_as_double((long long)((uint64_t)hi[0] << 32 | lo[0])), __longlong_as_double((long long)((uint64_t)hi[1] << 32 | lo[1])));
}
__device__ __forceinline__ int wave_min(int v) {
  uint32_t u = max16_u(~(uint32_t)v);
  auto w = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  u = max(w[0], w[1]);
  w = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return (int)~max(w[0], w[1]);
}

// One row by the whole wave with c in 64 bits.  The result is in lanes 0..15.
template <typename T>
__device__ __forceinline__ Pick select_wide(const SelectParams& p, int row, SelectScratch& scr) {
  const int lane = threadIdx.x & 63;
  const T* x = (const T*)p.logits + (size_t)row * p.ld;
  const double none = -(double)INFINITY;
  float v[4], b[4], m = -INFINITY;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = lane + 64 * i < p.E ? load_act(x, lane + 64 * i) : -INFINITY;
    b[i] = p.bias && lane + 64 * i < p.E ? p.bias[lane + 64 * i] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    nan |= v[i] != v[i];
    m = fmaxf(m, v[i]);
  }
  m = lanes_reduce<64, MaxOp>(m);
  if (!p.sigmoid) nan |= m == INFINITY;
  nan = __ballot(nan) != 0;
  m = m == -INFINITY ? 0.f : m;
  const bool sums = p.groups > 1 && p.best == 2, scored = (p.bias || sums) && !nan;
  // The candidates' c, or their logits where these have the same order, -inf and NaN being none.
#pragma unroll
  for (int i = 0; i < 4; ++i) scr.wide.c[lane + 64 * i] = v[i] > -INFINITY ? (double)v[i] : none;
  double total = 1.0;
  if (scored || !p.sigmoid) {
    total = 0.0;
#pragma unroll 1
    for (int e = lane; e < p.E; e += 64) {
      const double x = scr.wide.c[e];
      const double ex = exp(p.sigmoid ? -x : x - (double)m);
      scr.wide.group[e] = ex;
      total += ex;
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) total += __shfl_xor(total, o, 64);
  }
  if (scored) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = lane + 64 * i;
      if (e >= p.E) continue;
      const double ex = scr.wide.group[e];
      const double c = (p.sigmoid ? 1.0 : ex) / (p.sigmoid ? 1.0 + ex : total) + (double)b[i];
      if (scr.wide.c[e] != none) scr.wide.c[e] = c == c ? c : none;  // (NaN biases: below, a maximum is one of c)
    }
  }
  wave_sync();
  if (p.groups > 1) {
    const int size = p.E / p.groups;
#pragma unroll 1
    for (int g = lane; g < p.groups; g += 64) {
      double b1 = none, b2 = none;
#pragma unroll 8
      for (int e = g * size; e < (g + 1) * size; ++e) {
        const double c = scr.wide.c[e];
        b2 = c > b1 ? b1 : c > b2 ? c : b2;
        b1 = c > b1 ? c : b1;
      }
      scr.wide.group[g] = p.best == 2 && b2 != none ? b1 + b2 : b1;
    }
    wave_sync();
    uint32_t keep = 0;
#pragma unroll 1
    for (int g = lane, i = 0; g < p.groups; g += 64, ++i) {
      const double mine = scr.wide.group[g];
      int before = 0;
#pragma unroll 4
      for (int h = 0; h < p.groups; ++h) {
        const double o = scr.wide.group[h];
        before += o > mine || (o == mine && h < g);
      }
      keep |= (uint32_t)(before < p.top_groups) << i;
    }
    wave_sync();
    for (int g = lane, i = 0; g < p.groups; g += 64, ++i) scr.wide.group[g] = keep >> i & 1 ? 1.0 : 0.0;
    wave_sync();
#pragma unroll 1
    for (int e = lane; e < p.E; e += 64)
      if (scr.wide.group[e / size] == 0.0) scr.wide.c[e] = none;
    wave_sync();
  }
  double c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    c[i] = lane + 64 * i < p.E ? scr.wide.c[lane + 64 * i] : none;
    if (!p.bias && c[i] != none) c[i] = (double)v[i];  // (scores may have ended at 0 or 1, where logits differ)
  }
  int mine = -1;
#pragma unroll 1
  for (int j = 0; j < p.k; ++j) {
    const double top = wave_max64(fmax(fmax(c[0], c[1]), fmax(c[2], c[3])));
    if (top == none) break;
    int at = 1 << 20;
#pragma unroll
    for (int i = 3; i >= 0; --i) at = c[i] == top ? lane + 64 * i : at;
    at = wave_min(at);
    if (lane == j) mine = at;
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = lane + 64 * i == at ? none : c[i];
  }
  const Pick r = weigh(p, mine, mine >= 0 ? load_act(x, mine) : 0.f, m, p.sigmoid ? 1.f : (float)(1.0 / total), nan);
  wave_sync();
  return r;
}

__device__ __forceinline__ void order2(uint32_t& a, uint32_t& b) {
  const uint32_t hi = max(a, b);
  b = min(a, b);
  a = hi;
}
__device__ __forceinline__ void sort4(uint32_t* a) {
  order2(a[0], a[1]);
  order2(a[2], a[3]);
  order2(a[0], a[2]);
  order2(a[1], a[3]);
  order2(a[1], a[2]);
}
// Puts a sequence that falls and rises, or rises and falls, in descending order.
template <int N>
__device__ __forceinline__ void order_bitonic(uint32_t* a) {
#pragma unroll
  for (int d = N / 2; d >= 1; d >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i)
      if ((i & d) == 0) order2(a[i], a[i + d]);
}
// The largest N of two descending sequences of N, descending, in a.
template <int N>
__device__ __forceinline__ void merge_best(uint32_t* a, const uint32_t* b) {
#pragma unroll
  for (int i = 0; i < N; ++i) a[i] = max(a[i], b[N - 1 - i]);
  order_bitonic<N>(a);
}
// The largest of a lane's V keys, as many as are looked at, descending, in front.  Of 16 five: a row in
// 2500 has more of its 8 of 128 in one lane, with four one in 80, and such a row is done again.
template <int V>
constexpr int kDepth = V < 4 ? V : V < 16 ? 4 : 5;
template <int V>
__device__ __forceinline__ void best_keys(uint32_t (&a)[V]) {
  if constexpr (V >= 4) {
#pragma unroll
    for (int i = 0; i < V; i += 4) sort4(a + i);
  }
  if constexpr (V == 8) merge_best<4>(a, a + 4);
  if constexpr (V == 16) {
    // two fours, one of them turned round, to a descending eight
#pragma unroll
    for (int i = 0; i < 16; i += 8) {
      const uint32_t t4 = a[i + 4], t5 = a[i + 5];
      a[i + 4] = a[i + 7];
      a[i + 5] = a[i + 6];
      a[i + 6] = t5;
      a[i + 7] = t4;
      order_bitonic<8>(a + i);
    }
    merge_best<8>(a, a + 8);  // (what only places beyond the fifth need falls away)
  }
}

// The largest five of four pairs, each in order, descending, in front.
__device__ __forceinline__ void best_of_pairs(uint32_t* a) {
#pragma unroll
  for (int i = 0; i < 8; i += 4) {
    order2(a[i], a[i + 3]);
    order2(a[i + 1], a[i + 2]);
    order2(a[i], a[i + 1]);
    order2(a[i + 2], a[i + 3]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) order2(a[i], a[7 - i]);
  order_bitonic<4>(a);
  a[4] = max(max(a[4], a[5]), max(a[6], a[7]));
}

// c step + from is 2 (but for roundings, together less than 1) for the least c and below 2^24 for the largest.
__device__ __forceinline__ float fixed_step(float bias_max) { return 16777210.f / (1.f + 2.f * bias_max); }
__device__ __forceinline__ float fixed_from(float bias_max) { return fmaf(bias_max, fixed_step(bias_max), 2.f); }

// How far the fixed points of two candidates may be off (see select_rows), top being the largest score: four
// roundings and what is cut off beside the errors themselves.
__device__ __forceinline__ int score_margin(bool sigmoid, float top, float bias_max) {
  const float delta = (sigmoid ? 0x1p-21f : 0x1p-19f * top) + 0x1p-23f * (top + bias_max);
  return (int)fminf(2.f * delta * fixed_step(bias_max), 16777216.f) + 5;
}

__device__ __forceinline__ uint32_t order_key(float f) {
  const uint32_t u = __float_as_uint(f + 0.f);  // (-0 is 0)
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// Adds 1 to `before` for each of eight groups (their scores, all different, are in the row's lanes
// 0..7) that comes before the lane's own.
template <int H>
__device__ __forceinline__ void rank_step(int score, int& before) {
  before += (int)dpp_u<0x150 + H>((uint32_t)score) > score;  // lane H of each 16
  if constexpr (H + 1 < 8) rank_step<H + 1>(score, before);
}

// A row to each 16 lanes of the wave: its logits, expert l + 16 i to lane l, copies of the last behind it.
template <int V, typename T>
__device__ __forceinline__ void load_rows(const SelectParams& p, int row, float (&v)[V]) {
  int l = threadIdx.x & 15, E = p.E;
  asm volatile("" : "+v"(l), "+s"(E));  // (see select_rows)
  const T* x = (const T*)p.logits + (size_t)row * p.ld;
  // (No branch around a single load: each would be waited for before the next.)
  if (E == 16 * V) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = load_act(x, l + 16 * i);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = load_act(x, min(l + 16 * i, E - 1));
  }
}

// ... and its selection.  bias, as its fixed point, is in LDS, bias_max its largest magnitude.  *again:
// the row's result does not hold.
template <int V, typename T>
__device__ __forceinline__ Pick select_rows(const SelectParams& p, int row, bool live, float (&v)[V], const float* bias, float bias_max,
                                            SelectScratch& scr, bool* again) {
  const int lane = threadIdx.x & 63;
  // (What follows from these is worked out anew for every row: kept through the loop over rows, all of
  // it unrolled, it would fill the scalar registers and then vector ones.)
  int l = lane & 15, E = p.E, groups = p.groups, k = p.k;
  asm volatile("" : "+v"(l), "+s"(E), "+s"(groups), "+s"(k));
  const T* x = (const T*)p.logits + (size_t)row * p.ld;
  if (p.mask) live = live && p.mask[row] != 0;
  const bool sums = groups > 1 && p.best == 2, scored = p.bias || sums;
  const bool full = E == 16 * V;
  float any = 0.f;  // -inf or NaN, if one of the row's logits is
#pragma unroll
  for (int i = 0; i < V; ++i) any += v[i];
  if (!full) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = l + 16 * i < E ? v[i] : -INFINITY;
  }
  const bool holes = !full || __ballot(!(any > -INFINITY)) != 0;
  bool wide = any != any;
  // Fixed point of what is compared.  c = s + bias from 2 for the least that it can be (bias is held as
  // bias step + from); logits in steps of 2^-19 below the largest, down to 32 below.  Scores: with
  // t = x log2(e) rounded, 2^t is off by |t| half steps and a few; s (1 - s), or a share of the largest,
  // at most 2^-|t|, makes that less than 2^-22 of the largest score's whatever t.  The sum of a softmax
  // adds 20 half steps, which all have.  c is off by the addition's half step more: less than delta.
  constexpr float kLog2e = 1.44269502162933349609375f;
  const float step = fixed_step(bias_max);
  float m = 0.f, inv_sum = 1.f, top = 1.f;  // top: the largest score
  float c[V];
  if (p.sigmoid && scored) {
#pragma unroll
    for (int i = 0; i < V; ++i)
      c[i] = fmaf(__builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v[i] * -kLog2e)), step, bias[l + 16 * i]);
  } else {
    m = v[0];
#pragma unroll
    for (int i = 1; i < V; ++i) m = __builtin_amdgcn_fmed3f(m, v[i], INFINITY);  // the larger (fmaxf would first quiet both)
    m = lanes_reduce<16, MaxOp>(m);
    wide |= m == INFINITY;
    m = m == -INFINITY ? 0.f : m;
    if (!p.sigmoid && (scored || !p.renorm)) {  // (renormalised weights of the largest do not need the sum)
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        c[i] = __builtin_amdgcn_exp2f((v[i] - m) * kLog2e);
        sum += c[i];
      }
      sum = lanes_reduce<16, AddOp>(sum);
      inv_sum = top = sum == 0.f ? 0.f : __builtin_amdgcn_rcpf(sum);
    }
    if (scored) {
#pragma unroll
      for (int i = 0; i < V; ++i) c[i] = fmaf(c[i], inv_sum * step, bias[l + 16 * i]);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < V; ++i) c[i] = fmaxf(fmaf(v[i] - m, 0x1p19f, 16777215.f), 1.f);
    }
  }
  const int c_margin = score_margin(p.sigmoid, top, bias_max);
  const int margin = scored ? c_margin : sizeof(T) == 4 ? 4 : -1;
  uint32_t key[V];
  if (scored || sizeof(T) == 4) {
    if (holes) {  // 0, neither -inf nor NaN being candidates
#pragma unroll
      for (int i = 0; i < V; ++i) c[i] = v[i] > -INFINITY ? c[i] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = (uint32_t)c[i] << 8;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = v[i] > -INFINITY ? order_key(v[i]) & 0xFFFFFF00u : 0u;  // (16-bit logits are whole in 24 bits)
  }
#pragma unroll
  for (int i = 0; i < V; ++i) key[i] |= (uint32_t)(255 - l - 16 * i);
  if (holes) {
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = key[i] > 255u ? key[i] : 0u;
  }
  bool paired = false;  // the keys of the groups kept are four pairs in order, in front
  if (groups > 1) {
    // The groups' scores in the units of the keys; below all others (and so before none) where a
    // group has no expert left.
    const int base = sums ? (int)fixed_from(bias_max) : 0, size = E / groups;
    constexpr int kNone = -(1 << 25);
    auto part = [&](int i) { return key[i] >> 8; };
    auto score_of = [&](uint32_t b1, uint32_t b2) {
      return b1 == 0 ? kNone : (int)b1 + (sums && b2 != 0 ? (int)b2 - base : 0);
    };
    int least = -kNone, most = kNone;  // of the groups kept and dropped
    if (groups <= 8 && size % 16 == 0) {
      // a group is the same few of every lane's experts: lanes g and g + 8 find group g's best
      // two among those of eight lanes each
      const int each = size >> 4;
      int g = 0, left = each;
      uint32_t b1 = 0, b2 = 0;
      if (V == 16 && each == 2) {
#pragma unroll
        for (int i = 0; i + 1 < V; i += 2) {
          order2(key[i], key[i + 1]);
          scr.pair[i / 2][lane] = uint2{key[i], key[i + 1]};
        }
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          b2 = max(b2, min(b1, key[i]));
          b1 = max(b1, key[i]);
          if (--left == 0) {  // (the same for the whole wave)
            scr.pair[g++][lane] = uint2{b1, b2};
            b1 = b2 = 0;
            left = each;
          }
        }
      }
      wave_sync();
      const uint2* from8 = &scr.pair[l & 7][lane & 56];
      b1 = b2 = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint2 o = from8[i];
        const uint32_t lo = min(b1, o.x);
        b1 = max(b1, o.x);
        b2 = max(max(b2, o.y), lo);
      }
      {
        const uint32_t o1 = dpp_u<0x128>(b1), o2 = dpp_u<0x128>(b2);  // (row_ror 8)
        const uint32_t lo = min(b1, o1);
        b1 = max(b1, o1);
        b2 = max(max(b2, o2), lo);
      }
      wave_sync();
      // (the lower group first among equals; lanes of no group last)
      const int score = score_of(b1 >> 8, b2 >> 8);
      const int ranked = (l & 7) < groups ? score * 16 + 15 - (l & 7) : (2 * kNone - l) * 16;
      int before = 0;
      rank_step<0>(ranked, before);
      const bool in = before < p.top_groups;
      if ((l & 7) < groups) {
        if (in) least = score;
        else most = score;
      }
      const uint32_t keep = (uint32_t)(__ballot(in) >> (lane & 48));
      if (V == 16 && each == 2 && p.top_groups <= 4) {
        // half of the keys at most are left: as pairs from LDS they need not be sorted among 16 (131072 x
        // 256 in 8 groups, four kept: 68 us, 76 with the others masked)
        paired = true;
        uint32_t rest = keep & 255u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint2 o = scr.pair[__builtin_ctz(rest | 256u) & 7][lane];
          key[(2 * i) % V] = i < p.top_groups ? o.x : 0u;
          key[(2 * i + 1) % V] = i < p.top_groups ? o.y : 0u;
          rest &= rest - 1u;
        }
      } else {
        g = 0, left = each;
        uint32_t all = (uint32_t)__builtin_amdgcn_sbfe(keep, 0, 1);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          key[i] &= all;
          if (--left == 0) {
            left = each;
            all = (uint32_t)__builtin_amdgcn_sbfe(keep, ++g, 1);
          }
        }
      }
    } else {
      uint32_t* mine = scr.part[lane >> 4];
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (l + 16 * i < E) mine[l + 16 * i] = part(i);
      wave_sync();
      // lane l takes groups l, l + 16, ..; scores go where the first experts were: group g's start at g or later
#pragma unroll 1
      for (int g0 = 0; g0 < groups; g0 += 16) {
        const int g = g0 + l;
        uint32_t b1 = 0, b2 = 0;
        if (g < groups) {
#pragma unroll 4
          for (int e = g * size; e < (g + 1) * size; ++e) {
            const uint32_t o = mine[e];
            b2 = max(b2, min(b1, o));
            b1 = max(b1, o);
          }
        }
        wave_sync();
        if (g < groups) mine[g] = (uint32_t)score_of(b1, b2);
        wave_sync();
      }
      uint32_t keep = 0;
#pragma unroll 1
      for (int g = l, i = 0; g < groups; g += 16, ++i) {
        const int own = (int)mine[g];
        int before = 0;
#pragma unroll 4
        for (int h = 0; h < groups; ++h) {
          const int o = (int)mine[h];
          before += o > own || (o == own && h < g);
        }
        const bool in = before < p.top_groups;
        keep |= (uint32_t)in << i;
        if (in) least = min(least, own);
        else most = max(most, own);
      }
      wave_sync();
#pragma unroll 1
      for (int g = l, i = 0; g < groups; g += 16, ++i) mine[g] = keep >> i & 1;
      wave_sync();
      const uint32_t inv_size = 65536u / (uint32_t)size + 1u;  // e / size for e < 256
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const uint32_t g = min((uint32_t)(l + 16 * i) * inv_size >> 16, (uint32_t)groups - 1);
        if (mine[g] == 0) key[i] = 0u;
      }
      wave_sync();
    }
    least = (int)(~max16_u(~((uint32_t)least ^ 0x80000000u)) ^ 0x80000000u);
    most = (int)(max16_u((uint32_t)most ^ 0x80000000u) ^ 0x80000000u);
    // (two sums of two, and the unit that `base` is off)
    const int group_margin = sums ? 2 * c_margin + 2 : margin;
    wide |= most > kNone && least - most <= group_margin;
  }
  if constexpr (V == 16) {
    if (paired) best_of_pairs(key);
    else best_keys<V>(key);
  } else {
    best_keys<V>(key);
  }
  constexpr int D = kDepth<V>;
  const uint32_t last = key[D - 1];
  uint32_t mine = 0, next = 0;
  for (int j = 0; j <= k; ++j) {
    const uint32_t top_key = max16_u(key[0]);
    if (l == j) mine = top_key;
    next = top_key;  // in the end the first that is not selected
    const bool won = key[0] == top_key;
#pragma unroll
    for (int i = 0; i + 1 < D; ++i) key[i] = won ? key[i + 1] : key[i];
    key[D - 1] = won ? 0u : key[D - 1];
  }
  if (V > D) wide |= key[0] == 0u && last != 0u;  // a lane may have had more
  const uint32_t right = dpp_u<0x101>(mine);  // (row_shl 1: the next lane's, read by all lanes)
  const uint32_t after = l == k - 1 ? next : right;
  const int e = l < k && mine != 0u ? 255 - (int)(mine & 255u) : -1;
  const float of_e = e >= 0 ? load_act(x, e) : 0.f;
  // among the selected, logits themselves tell without a bias whether their order is right
  const float of_right = dpp<0x101>(of_e);
  const int e_right = (int)dpp_u<0x101>((uint32_t)e);
  bool order = (int)(mine >> 8) - (int)(after >> 8) > margin;
  if (!p.bias && l < k - 1) order = of_e > of_right || (of_e == of_right && e < e_right);
  wide |= e >= 0 && after != 0u && !order;
  *again = (__ballot(wide && live) >> (lane & 48) & 0xFFFFu) != 0;
  return weigh(p, live ? e : -1, of_e, m, inv_sum, false);
}

// Of long batches of up to 16 experts and four selected a row is one lane's, which sorts all of its keys: the
// same comparisons and, sums being taken in the same order, the same bits as of select_rows, in a tenth of its
// instructions.
constexpr int kLaneMost = 4;
template <int V, typename T>
__device__ __forceinline__ bool select_lane(const SelectParams& p, int row, bool live, const float* bias, float bias_max, Pick (&r)[kLaneMost]) {
  const T* x = (const T*)p.logits + (size_t)row * p.ld;
  float v[V], c[V], any = 0.f;
  if (p.E == V) {
#pragma unroll
    for (int i = 0; i < V; i += 8) {
      float o[8];
      load_n(x + i, o);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i + j] = o[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = load_act(x, min(i, p.E - 1));
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    any += v[i];
    v[i] = i < p.E ? v[i] : -INFINITY;
  }
  bool wide = any != any;
  constexpr float kLog2e = 1.44269502162933349609375f;
  const float step = fixed_step(bias_max);
  float m = 0.f, inv_sum = 1.f, top = 1.f;
  if (p.sigmoid && p.bias) {
#pragma unroll
    for (int i = 0; i < V; ++i) c[i] = fmaf(__builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v[i] * -kLog2e)), step, bias[i]);
  } else {
    m = v[0];
#pragma unroll
    for (int i = 1; i < V; ++i) m = __builtin_amdgcn_fmed3f(m, v[i], INFINITY);
    wide |= m == INFINITY;
    m = m == -INFINITY ? 0.f : m;
    if (!p.sigmoid && (p.bias || !p.renorm)) {
      float sum[V];
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] = c[i] = __builtin_amdgcn_exp2f((v[i] - m) * kLog2e);
#pragma unroll
      for (int d = 1; d < V; d *= 2)
#pragma unroll
        for (int i = 0; i < V; i += 2 * d) sum[i] += sum[i + d];
      inv_sum = top = sum[0] == 0.f ? 0.f : __builtin_amdgcn_rcpf(sum[0]);
    }
    if (p.bias) {
#pragma unroll
      for (int i = 0; i < V; ++i) c[i] = fmaf(c[i], inv_sum * step, bias[i]);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < V; ++i) c[i] = fmaxf(fmaf(v[i] - m, 0x1p19f, 16777215.f), 1.f);
    }
  }
  const int margin = p.bias ? score_margin(p.sigmoid, top, bias_max) : sizeof(T) == 4 ? 4 : -1;
  uint32_t best[kLaneMost + 1] = {};
#pragma unroll
  for (int i = 0; i < V; ++i) {
    uint32_t key = p.bias || sizeof(T) == 4 ? (uint32_t)c[i] << 8 : order_key(v[i]) & 0xFFFFFF00u;
    key = v[i] > -INFINITY ? key | (uint32_t)(255 - i) : 0u;
    key = key > 255u ? key : 0u;
#pragma unroll
    for (int j = 0; j <= kLaneMost; ++j) order2(best[j], key);
  }
  float of[kLaneMost + 1];
#pragma unroll
  for (int j = 0; j < kLaneMost; ++j) {
    r[j].e = j < p.k && best[j] != 0u ? 255 - (int)(best[j] & 255u) : -1;
    of[j] = r[j].e >= 0 ? load_act(x, r[j].e) : 0.f;
  }
#pragma unroll
  for (int j = 0; j < kLaneMost; ++j) {
    bool order = (int)(best[j] >> 8) - (int)(best[j + 1] >> 8) > margin;
    if (j + 1 < kLaneMost && !p.bias && j < p.k - 1) order = of[j] > of[j + 1] || (of[j] == of[j + 1] && r[j].e < r[j + 1].e);
    wide |= r[j].e >= 0 && best[j + 1] != 0u && !order;
  }
#pragma unroll
  for (int j = 0; j < kLaneMost; ++j) {
    if (!live) r[j].e = -1;
    r[j].w = r[j].e < 0 ? 0.f : p.sigmoid ? sigmoid(of[j]) : exp_neg(of[j] - m) * inv_sum;
  }
  const float total = (r[0].w + r[1].w) + (r[2].w + r[3].w);
  const float scale = p.renorm ? p.scale * __builtin_amdgcn_rcpf(total + kTiny) : p.scale;
#pragma unroll
  for (int j = 0; j < kLaneMost; ++j) r[j].w = r[j].e < 0 ? 0.f : r[j].w * scale;
  return wide && live;
}

// Of long batches of 17 to 64 experts and eight selected a row is four lanes', experts 16 i + 4 q + 0 .. 3 of
// lane q's: each sorts its largest eight, which then meet in twice two, and so all have the row's, and in `next`
// the ninth.  Comparisons, sums' order and bits are those of select_rows here too.  Lane q has picks q and q + 4.
constexpr int kQuadMost = 8;
__device__ __forceinline__ uint32_t of4(int q, uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return q & 2 ? (q & 1 ? d : c) : (q & 1 ? b : a); }
__device__ __forceinline__ void order_eight(uint32_t* a) {  // of two fours in order
  const uint32_t t4 = a[4], t5 = a[5];
  a[4] = a[7];
  a[5] = a[6];
  a[6] = t5;
  a[7] = t4;
  order_bitonic<8>(a);
}
// The largest eight of two eights in order to a, in order; the largest of the others to next.
__device__ __forceinline__ void meet_eights(uint32_t* a, const uint32_t (&o)[8], uint32_t& next) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    next = max(next, min(a[i], o[7 - i]));
    a[i] = max(a[i], o[7 - i]);
  }
  order_bitonic<8>(a);
}
template <int CTRL>
__device__ __forceinline__ void meet_lanes(uint32_t* a, uint32_t& next) {
  uint32_t o[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = dpp_u<CTRL>(a[i]);
  next = max(next, dpp_u<CTRL>(next));
  meet_eights(a, o, next);
}
template <typename T>
__device__ __forceinline__ bool select_quad(const SelectParams& p, int row, bool live, const float* bias, float bias_max, Pick (&r)[2]) {
  const int lane = threadIdx.x & 63, q = lane & 3;
  const T* x = (const T*)p.logits + (size_t)row * p.ld;
  float v[16], c[16], any = 0.f;
  if (p.E == 64) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float o[4];
      load_n(x + 16 * i + 4 * q, o);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[4 * i + j] = o[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = load_act(x, min(16 * (i >> 2) + 4 * q + (i & 3), p.E - 1));
  }
  auto expert = [&](int i) { return 16 * (i >> 2) + 4 * q + (i & 3); };
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    any += v[i];
    v[i] = expert(i) < p.E ? v[i] : -INFINITY;
  }
  bool wide = any != any;
  constexpr float kLog2e = 1.44269502162933349609375f;
  const float step = fixed_step(bias_max);
  float m = 0.f, inv_sum = 1.f, top = 1.f;
  if (p.sigmoid && p.bias) {
#pragma unroll
    for (int i = 0; i < 16; ++i) c[i] = fmaf(__builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v[i] * -kLog2e)), step, bias[expert(i)]);
  } else {
    m = v[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) m = __builtin_amdgcn_fmed3f(m, v[i], INFINITY);
    m = lanes_reduce<4, MaxOp>(m);
    wide |= m == INFINITY;
    m = m == -INFINITY ? 0.f : m;
    if (!p.sigmoid && (p.bias || !p.renorm)) {
      float sum[4];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        c[i] = __builtin_amdgcn_exp2f((v[i] - m) * kLog2e);
        sum[i & 3] = i < 4 ? c[i] : sum[i & 3] + c[i];
      }
      const float all = lanes_reduce<4, AddOp>((sum[0] + sum[1]) + (sum[2] + sum[3]));
      inv_sum = top = all == 0.f ? 0.f : __builtin_amdgcn_rcpf(all);
    }
    if (p.bias) {
#pragma unroll
      for (int i = 0; i < 16; ++i) c[i] = fmaf(c[i], inv_sum * step, bias[expert(i)]);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 16; ++i) c[i] = fmaxf(fmaf(v[i] - m, 0x1p19f, 16777215.f), 1.f);
    }
  }
  const int margin = p.bias ? score_margin(p.sigmoid, top, bias_max) : sizeof(T) == 4 ? 4 : -1;
  uint32_t key[16], next = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t part = p.bias || sizeof(T) == 4 ? (uint32_t)c[i] << 8 : order_key(v[i]) & 0xFFFFFF00u;
    key[i] = v[i] > -INFINITY && part != 0u ? part | (uint32_t)(255 - expert(i)) : 0u;
  }
#pragma unroll
  for (int i = 0; i < 16; i += 4) sort4(key + i);
  order_eight(key);
  order_eight(key + 8);
  {
    uint32_t o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = key[8 + i];
    meet_eights(key, o, next);
  }
  meet_lanes<0xB1>(key, next);  // quad_perm 1,0,3,2
  meet_lanes<0x4E>(key, next);  // quad_perm 2,3,0,1
  const uint32_t mine[2] = {of4(q, key[0], key[1], key[2], key[3]), of4(q, key[4], key[5], key[6], key[7])};
  const uint32_t after[2] = {of4(q, key[1], key[2], key[3], key[4]), of4(q, key[5], key[6], key[7], next)};
  float of[2], right[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    r[u].e = q + 4 * u < p.k && mine[u] != 0u ? 255 - (int)(mine[u] & 255u) : -1;
    of[u] = r[u].e >= 0 ? load_act(x, r[u].e) : 0.f;
  }
  right[0] = dpp<0x39>(of[0]);  // quad_perm 1,2,3,0
  right[1] = dpp<0x39>(of[1]);
  if (q == 3) right[0] = right[1];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    bool order = (int)(mine[u] >> 8) - (int)(after[u] >> 8) > margin;
    if (!p.bias && q + 4 * u < p.k - 1) order = of[u] > right[u] || (of[u] == right[u] && r[u].e < 255 - (int)(after[u] & 255u));
    wide |= r[u].e >= 0 && after[u] != 0u && !order;
    if (!live) r[u].e = -1;
    r[u].w = r[u].e < 0 ? 0.f : p.sigmoid ? sigmoid(of[u]) : exp_neg(of[u] - m) * inv_sum;
  }
  float scale = p.scale;
  if (p.renorm) scale *= __builtin_amdgcn_rcpf(lanes_reduce<4, AddOp>(r[0].w) + lanes_reduce<4, AddOp>(r[1].w) + kTiny);
#pragma unroll
  for (int u = 0; u < 2; ++u) r[u].w = r[u].e < 0 ? 0.f : r[u].w * scale;
  return (__ballot(wide && live) >> (lane & 60) & 15u) != 0;
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

constexpr int kHeld = 2;  // pairs that a thread keeps from marking them to placing them
struct PlaceLds {
  uint32_t bits[MIRA_MAX_EXPERTS][kWords];
  int base[MIRA_MAX_EXPERTS];
  int wave_sums[4];
};

// Order and positions of a chunk's pairs, by the whole workgroup.  sel(i) is the expert
// of pair i of the chunk, kept(t) whether its token t has shared experts; thread g's `of` has the pairs of
// group g in earlier chunks (x) and in the call (y).
template <int THREADS, typename Sel, typename Kept>
__device__ __forceinline__ void place_pairs(const SelectParams& p, PlaceLds& L, int chunk, Sel sel, Kept kept, int2 of) {
  const int t = threadIdx.x, G = p.E + p.S, t0 = chunk * p.chunk, n = min(p.chunk, p.T - t0);
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
  int held_g[kHeld], held_tok[kHeld];  // a thread's first pairs, loaded beside the counts
#pragma unroll
  for (int u = 0; u < kHeld; ++u) {
    held_g[u] = -1;
    if (t + u * THREADS < pairs) held_g[u] = pair_of(t + u * THREADS, &held_tok[u]);
  }
  for (int i = t; i < G * kWords; i += THREADS) (&L.bits[0][0])[i] = 0;
  int all;
  const int mine = t < G ? of.y : 0;
  const int off = scan256(mine, L.wave_sums, &all);  // (its barrier: the bits are zero)
  if (t < G) {
    L.base[t] = off + of.x;
    if (chunk == 0) {
      if (p.counts_out) p.counts_out[t] = mine;
      if (p.offsets_out) p.offsets_out[t] = off;
    }
  }
  if (chunk == 0 && t == 0 && p.offsets_out) p.offsets_out[G] = all;
  auto mark = [&](int g, int tok) {
    if (g >= 0) atomicOr(&L.bits[g][tok >> 5], 1u << (tok & 31));
  };
#pragma unroll
  for (int u = 0; u < kHeld; ++u) mark(held_g[u], held_tok[u]);
  for (int i = t + kHeld * THREADS; i < pairs; i += THREADS) {
    int tok;
    const int g = pair_of(i, &tok);
    mark(g, tok);
  }
  __syncthreads();
  const size_t P = (size_t)p.T * (p.k + p.S), Tk = (size_t)p.T * p.k;
  auto put = [&](int i, int g, int tok) {
    const size_t pair = i < routed ? (size_t)t0 * p.k + i : Tk + (size_t)((i - routed) / n) * p.T + t0 + tok;
    int at = -1;
    if (g >= 0) {
      at = L.base[g] + __popc(L.bits[g][tok >> 5] & ((1u << (tok & 31)) - 1u));
      for (int w = 0; w < (tok >> 5); ++w) at += __popc(L.bits[g][w]);
      if (p.order) p.order[at] = (int)pair;
    }
    if (p.pos) p.pos[pair] = at;
  };
#pragma unroll
  for (int u = 0; u < kHeld; ++u)
    if (t + u * THREADS < pairs) put(t + u * THREADS, held_g[u], held_tok[u]);
  for (int i = t + kHeld * THREADS; i < pairs; i += THREADS) {
    int tok;
    const int g = pair_of(i, &tok);
    put(i, g, tok);
  }
  if (p.order)
    for (size_t i = (size_t)all + (size_t)chunk * THREADS + t; i < P; i += (size_t)p.chunks * THREADS) p.order[i] = -1;
}

// A chunk of tokens: a wave takes four rows at a time, then the rows that are to be done again, one by
// one (within the loop the constants of a 64-bit exp would be held through it).  Registers are one number for the
// whole kernel: up to 128 experts by 16 lanes and by one it is the 64-bit rows' (93 and 105; 57 to 70 and 38 to 75
// without them), by four and above 128 experts the loop's.  LANES of 4 and 1: rows of 4 lanes, or of one.
// One chunk places its pairs at once (ONE); several leave their counts.
template <int V, bool ONE, int LANES, typename T>
__global__ __launch_bounds__(ONE ? kOneThreads : LANES == 1 ? kChunk : kThreads, LANES == 4 ? 4 : 1) void route_select_kernel(SelectParams p) {
  constexpr int kWaves = (ONE ? kOneThreads : LANES == 1 ? kChunk : kThreads) / 64;
  __shared__ SelectScratch scr[kWaves];
  __shared__ float bias[MIRA_MAX_EXPERTS];
  __shared__ float wave_max_bias[4];
  __shared__ int hist[MIRA_MAX_EXPERTS];
  __shared__ int kept, n_again;
  __shared__ uint8_t rows_again[kChunk];
  __shared__ int16_t sel[ONE ? kChunk * MIRA_MAX_TOPK : 1];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, l = lane & 15;
  const int t0 = blockIdx.x * p.chunk, n = min(p.chunk, p.T - t0);
  if (t < MIRA_MAX_EXPERTS) {
    hist[t] = 0;
    bias[t] = p.bias && t < p.E ? p.bias[t] : 0.f;
    const float b = lanes_reduce<64, MaxOp>(fabsf(bias[t]));
    if (lane == 0) wave_max_bias[wave] = b;
  }
  if (t == 0) kept = n_again = 0;
  __syncthreads();
  const float bias_max = fmaxf(fmaxf(wave_max_bias[0], wave_max_bias[1]), fmaxf(wave_max_bias[2], wave_max_bias[3]));
  if (t < MIRA_MAX_EXPERTS) bias[t] = fmaf(bias[t], fixed_step(bias_max), fixed_from(bias_max));
  __syncthreads();
  auto write = [&](int i, const Pick& r) {  // lane l of a row's lanes
    if (l >= p.k) return;
    const size_t at = (size_t)(t0 + i) * p.k + l;
    p.idx[at] = r.e;
    if (p.weight) p.weight[at] = r.w;
    if (p.place) {
      if (ONE) sel[i * p.k + l] = (int16_t)r.e;
      if (r.e >= 0) atomicAdd(&hist[r.e], 1);
    }
  };
  if constexpr (LANES == 4) {
    for (int i0 = wave * 16; i0 < n; i0 += kWaves * 16) {
      const int i = i0 + (lane >> 2), q = lane & 3;
      const bool in = i < n, live = in && (!p.mask || p.mask[t0 + min(i, n - 1)] != 0);
      Pick r[2];
      const bool again = select_quad<T>(p, t0 + min(i, n - 1), live, bias, bias_max, r);
      if (!in) continue;
      if (again && q == 0) rows_again[atomicAdd(&n_again, 1)] = (uint8_t)i;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (again || q + 4 * u >= p.k) continue;
        const size_t at = (size_t)(t0 + i) * p.k + q + 4 * u;
        p.idx[at] = r[u].e;
        if (p.weight) p.weight[at] = r[u].w;
        if (p.place && r[u].e >= 0) atomicAdd(&hist[r[u].e], 1);
      }
      if (p.place && live && q == 0) atomicAdd(&kept, 1);
    }
  }
  if constexpr (LANES == 1) {  // (a chunk has a thread for each of its tokens at most)
    if (t < n) {
      const bool live = !p.mask || p.mask[t0 + t] != 0;
      Pick r[kLaneMost];
      if (select_lane<V, T>(p, t0 + t, live, bias, bias_max, r)) {
        rows_again[atomicAdd(&n_again, 1)] = (uint8_t)t;
      } else {
        const size_t at = (size_t)(t0 + t) * p.k;
#pragma unroll
        for (int j = 0; j < kLaneMost; ++j) {
          if (j >= p.k) continue;
          p.idx[at + j] = r[j].e;
          if (p.weight) p.weight[at + j] = r[j].w;
          if (p.place && r[j].e >= 0) atomicAdd(&hist[r[j].e], 1);
        }
      }
      if (p.place && live) atomicAdd(&kept, 1);
    }
  }
  for (int i0 = LANES < 16 ? n : wave * 4; i0 < n; i0 += kWaves * 4) {
    const int i = i0 + (lane >> 4);
    const bool live = i < n;
    float v[V];
    load_rows<V, T>(p, t0 + min(i, n - 1), v);
    bool again;
    const Pick r = select_rows<V, T>(p, t0 + min(i, n - 1), live, v, bias, bias_max, scr[wave], &again);
    if (live) {
      if (!again) write(i, r);
      else if (l == 0) rows_again[atomicAdd(&n_again, 1)] = (uint8_t)i;
      if (p.place && l == 0 && (!p.mask || p.mask[t0 + i])) atomicAdd(&kept, 1);
    }
  }
  __syncthreads();
  const int redo = n_again;
  for (int j = wave; j < redo; j += kWaves) {
    const int i = rows_again[j];
    const Pick r = select_wide<T>(p, t0 + i, scr[wave]);
    if (lane < 16) write(i, r);
  }
  if (!p.place) return;
  __syncthreads();
  auto count = [&](int g) { return g < p.E ? hist[g] : kept; };
  if constexpr (ONE) {
    __shared__ PlaceLds place;
    place_pairs<kOneThreads>(p, place, 0, [&](int i) { return (int)sel[i]; }, [&](int i) { return !p.mask || p.mask[i] != 0; },
                             int2{0, t < p.E + p.S ? count(t) : 0});
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

// Places a chunk's pairs.  FEW: the chunks' counts are added up here, by as many threads to a group as
// there are for the next power of two of groups.
template <bool FEW>
__global__ __launch_bounds__(kPlaceThreads) void route_place_kernel(SelectParams p, int log_groups) {
  __shared__ PlaceLds place;
  __shared__ int2 part[FEW ? kPlaceThreads : 1];  // pairs of earlier chunks, of all
  const int chunk = blockIdx.x, t0 = chunk * p.chunk, t = threadIdx.x, G = p.E + p.S;
  int2 of{0, 0};  // of group t
  if constexpr (FEW) {
    const int g = t & ((1 << log_groups) - 1), many = kPlaceThreads >> log_groups;
    int2 s{0, 0};
    if (log_groups < 6) {  // a wave's threads of the same group first (131072 of 4 of 13: 16.6 us, 17.3 all through LDS)
      if (g < G) {
        for (int c0 = t >> log_groups; c0 < p.chunks; c0 += 8 * many) {
          int v[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) v[u] = p.counts[min(c0 + u * many, p.chunks - 1) * G + g];  // (below 2^15)
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const int c = c0 + u * many;
            s.x += c < chunk ? v[u] : 0;
            s.y += c < p.chunks ? v[u] : 0;
          }
        }
      }
      for (int o = 1 << log_groups; o < 64; o *= 2) {  // (a wave's threads of the same group)
        s.x += __shfl_xor(s.x, o, 64);
        s.y += __shfl_xor(s.y, o, 64);
      }
      if ((t & 63) < 1 << log_groups) part[((t >> 6) << log_groups) + (t & 63)] = s;
    } else {  // (eight loads at once as the compiler arranges them: 16384 of 6 of 64 and 2 13.6 us, 14.4 as above)
      if (g < G) {
#pragma unroll 8
        for (int c = t >> log_groups; c < p.chunks; c += many) {
          const int v = p.counts[c * G + g];
          s.x += c < chunk ? v : 0;
          s.y += v;
        }
      }
      part[t] = s;
    }
    __syncthreads();
    if (t < G)
      for (int i = 0; i < min(many, kPlaceThreads / 64); ++i) {
        const int2 o = part[(i << log_groups) + t];
        of.x += o.x;
        of.y += o.y;
      }
  } else if (t < G) {
    of = int2{p.counts[(size_t)chunk * G + t], p.totals[t]};
  }
  const int32_t* idx = p.idx + (size_t)t0 * p.k;
  place_pairs<kPlaceThreads>(
      p, place, chunk, [&](int i) { return (int)idx[i]; }, [&](int i) { return !p.mask || p.mask[t0 + i] != 0; }, of);
}

// Most tokens of a call in one launch, a workgroup of 64 rows at a time (us, in one against two: 64 of
// 256 experts 7.6 and 9.0, 96 8.8 and 9.0, 128 11.2 and 9.1, of 64 experts 7.8 and 9.0).
int one_tokens(int E) { return E <= 64 ? 128 : 64; }

// Tokens of a chunk: 32 until the chunks fill the CUs, then more, in steps of 32.
int chunk_tokens(int T, int E) {
  if (T <= one_tokens(E)) return one_tokens(E);
  const int c = ((T + 255) / 256 + 31) / 32 * 32;
  return c < 32 ? 32 : c > kChunk ? kChunk : c;
}
int chunk_count(int T, int E) { return (int)(((int64_t)T + chunk_tokens(T, E) - 1) / chunk_tokens(T, E)); }

template <int V, typename T>
void launch_select(const SelectParams& p, hipStream_t st) {
  launch_timed("route_select", p.chunks == 1 ? route_select_kernel<V, true, 16, T> : route_select_kernel<V, false, 16, T>, dim3(p.chunks),
               dim3(p.chunks == 1 ? kOneThreads : kThreads), 0, st, p);
}

// Tokens from which on rows of up to 64 experts are four lanes' or one's.  us by 16 lanes and by four: 131072 of 6 of 64 and 2 shared
// 33.7 and 27.0, of 8 of 64 bf16 with bias 37.6 and 29.7, 9000 of 6 of 64 and 2 12.8 and 12.1, of 2 of 17 9.0 and 8.7.
// By 16 and by one: 131072 of 2 of 8 21.3 and 12.5, of 4 of 13 bf16 with bias and mask 25.4 and 17.4; 12000 9.5 and
// 8.7, 11.9 and 11.8; 8192 8.7 and 9.2, 10.7 and 12.1.
constexpr int kLaneTokens = 8192;

template <typename T>
void launch_select_of(const SelectParams& p, hipStream_t st) {
  if (p.E <= 16 && p.k <= kLaneMost && p.groups == 1 && p.T > kLaneTokens)
    launch_timed("route_select", p.E <= 8 ? route_select_kernel<8, false, 1, T> : route_select_kernel<16, false, 1, T>, dim3(p.chunks),
                 dim3(kChunk), 0, st, p);
  else if (p.E <= 64 && p.k <= kQuadMost && p.groups == 1 && p.T > kLaneTokens)
    launch_timed("route_select", route_select_kernel<4, false, 4, T>, dim3(p.chunks), dim3(kThreads), 0, st, p);
  else if (p.E <= 16) launch_select<1, T>(p, st);
  else if (p.E <= 64) launch_select<4, T>(p, st);
  else if (p.E <= 128) launch_select<8, T>(p, st);
  else launch_select<16, T>(p, st);
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

// Four values of a row from column c on; a lane at the row's end loads its last four and settle4(), called
// once all loads are on their way, moves them to their places.
template <typename T>
__device__ __forceinline__ void load4(const T* row, int c, int cols, float (&v)[4]) {
  if (cols >= 4) {  // (the same for all)
    load_n(row + min(c, cols - 4), v);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = c + i < cols ? load_act(row, c + i) : 0.f;
  }
}
__device__ __forceinline__ void settle4(float (&v)[4], int c, int cols, float beyond) {
  if (c + 4 <= cols) return;
  if (cols >= 4) {
    const int n = c + 4 - cols;
    if (n & 2) v[0] = v[2], v[1] = v[3];
    if (n & 1) v[0] = v[1], v[1] = v[2], v[2] = v[3];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = c + i < cols ? v[i] : beyond;
}
typedef uint32_t v2u_any __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ void store4(float* row, int c, int cols, const float (&v)[4]) {
  if (c + 4 <= cols) {
    *(v4f_any*)(row + c) = v4f{v[0], v[1], v[2], v[3]};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i < cols) row[c + i] = v[i];
  }
}
__device__ __forceinline__ void store4(uint16_t* row, int c, int cols, const float (&v)[4]) {
  if (c + 4 <= cols) {
    *(v2u_any*)(row + c) = v2u_any{to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3])};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i < cols) row[c + i] = to_bf16(v[i]);
  }
}

// Adds what selection J of k, in lane J of each 16, has for a lane's experts, c + 64 q + i, and (N)
// counts it.
template <int J, bool N, int Q>
__device__ __forceinline__ void spread(int sel, float g, int k, int c, float (&sum)[Q][4], float (&n)[Q][4]) {
  if (J < k) {  // (the same for the whole wave)
    const int at = (int)dpp_u<0x150 + J>((uint32_t)sel) - c;
    const float of = dpp<0x150 + J>(g);
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sum[q][i] += at == 64 * q + i ? of : 0.f;
        if (N) n[q][i] += at == 64 * q + i ? 1.f : 0.f;
      }
    if constexpr (J + 1 < MIRA_MAX_TOPK) spread<J + 1, N, Q>(sel, g, k, c, sum, n);
  }
}

// A row to 16 lanes, experts 4 l + 64 q + 0 .. 3 to lane l; lane j has selection j.
//   ds_e = scale (g_e - [renorm] A / D) / D on the selected, A = sum g s, D = sum s + 1e-20 (1 without renorm);
//   sigmoid: dl_e = ds_e s_e (1 - s_e), of the selected logits alone;  softmax: dl_e = s_e (ds_e - B), B = sum
//   ds s, which with renorm is scale (A / D) (1e-20 / D): as a difference of its terms nothing of it
//   would be left.
// 131072 x 256 fp32 softmax 65 us for 276 MB (4.3 TB/s; a copy takes 54: 119 registers leave four waves a SIMD to
// cover the loads), sigmoid 46 us for 147 MB (the selected logits are lines of their own). A row to 64 lanes, one
// in turn, waited for its loads three times a row (89 and 72 us).
template <int Q, typename T>
__global__ __launch_bounds__(256) void route_select_grad_kernel(SelectGradParams p) {
  const int l = threadIdx.x & 15, c = 4 * l;
  // (whole groups of lanes leave the loop)
  for (size_t row = (size_t)blockIdx.x * 16 + (threadIdx.x >> 4); row < (size_t)p.T; row += (size_t)gridDim.x * 16) {
    const T* x = (const T*)p.logits + row * p.ld;
    float v[Q][4], o[Q][4], n[Q][4];
    int sel = -1;
    if (l < p.k) sel = p.idx[row * p.k + l];
    if (!p.sigmoid) {
#pragma unroll
      for (int q = 0; q < Q; ++q) load4(x, c + 64 * q, p.E, v[q]);
    }
    float add[Q][4];
    if (p.add) {
#pragma unroll
      for (int q = 0; q < Q; ++q) load4((const T*)p.add + row * p.ld_add, c + 64 * q, p.E, add[q]);
    }
    if ((uint32_t)sel >= (uint32_t)p.E) sel = -1;
    float g = sel >= 0 ? p.dweight[row * p.k + l] : 0.f;
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[q][i] = n[q][i] = 0.f;
    if (p.sigmoid) {
      float s = 0.f, rest = 0.f;
      if (sel >= 0) {
        const float u = load_act(x, sel), e = exp_neg(-fabsf(u)), r = __builtin_amdgcn_rcpf(1.f + e);
        s = u >= 0.f ? r : e * r;
        rest = u >= 0.f ? e * r : r;
        if (u == -INFINITY) sel = -1, g = s = 0.f;  // (no entry, whatever arrives at it)
      }
      const float A = lanes_reduce<16, AddOp>(g * s), D = lanes_reduce<16, AddOp>(s) + kTiny;
      const float inv = p.renorm ? 1.f / D : 1.f, mean = p.renorm ? A * inv : 0.f;
      spread<0, false, Q>(sel, sel >= 0 ? p.scale * inv * (g - mean) * s * rest : 0.f, p.k, c, o, n);
    } else {
      // Entries of experts of -inf are none.  Only a wave whose rows have such logits looks which those are (looked up in
      // every row: 30011 x 61 bf16 7.2 us, 6.8 so).
      float least[4] = {v[0][0], v[0][1], v[0][2], v[0][3]};  // -inf or NaN, if one of the lane's logits is
#pragma unroll
      for (int q = 1; q < Q; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i) least[i] += v[q][i];
      if (__ballot(!((least[0] + least[1]) + (least[2] + least[3]) > -INFINITY)) && sel >= 0 && load_act(x, sel) == -INFINITY) sel = -1, g = 0.f;
      if (p.renorm) spread<0, true, Q>(sel, g, p.k, c, o, n);
      else spread<0, false, Q>(sel, g, p.k, c, o, n);
      float m = -INFINITY;
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        settle4(v[q], c + 64 * q, p.E, -INFINITY);
        m = fmaxf(m, fmaxf(fmaxf(v[q][0], v[q][1]), fmaxf(v[q][2], v[q][3])));
      }
      m = lanes_reduce<16, MaxOp>(m);
      m = m == -INFINITY ? 0.f : m;
      float sum = 0.f, A = 0.f, D = 0.f;
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[q][i] = exp_neg(v[q][i] - m);
          sum += v[q][i];
          A = fmaf(o[q][i], v[q][i], A);
          D = fmaf(n[q][i], v[q][i], D);
        }
      sum = lanes_reduce<16, AddOp>(sum);
      const float to_score = sum == 0.f ? 0.f : __builtin_amdgcn_rcpf(sum);
      A = lanes_reduce<16, AddOp>(A) * to_score;
      D = lanes_reduce<16, AddOp>(D) * to_score + kTiny;
      const float inv = p.renorm ? 1.f / D : 1.f, mean = p.renorm ? A * inv : 0.f;
      const float B = p.scale * (p.renorm ? mean * (kTiny * inv) : A);
      const bool any = lanes_reduce<16, MaxOp>(sel >= 0 ? 1.f : 0.f) > 0.f;
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          o[q][i] = any ? v[q][i] * to_score * (p.scale * inv * (o[q][i] - n[q][i] * mean) - B) : 0.f;
    }
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if (p.add) {
        settle4(add[q], c + 64 * q, p.E, 0.f);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[q][i] += add[q][i];
      }
      store4((T*)p.d + row * p.ld_d, c + 64 * q, p.E, o[q]);
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
  const size_t chunks = T <= 8192 ? ((size_t)T + 31) / 32 : T <= 256 * kChunk ? 256 : ((size_t)T + kChunk - 1) / kChunk;
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
  p.chunk = chunk_tokens(p.T, p.E);
  p.chunks = p.T < 1 ? 1 : chunk_count(p.T, p.E);
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
    int log_groups = 4;
    while (1 << log_groups < G) ++log_groups;
    if ((int64_t)p.chunks * G <= kFewCounts) {
      launch_timed("route_place", route_place_kernel<true>, dim3(p.chunks), dim3(kPlaceThreads), 0, st, p, log_groups);
    } else {
      launch_timed("route_scan", route_scan_kernel, dim3(G), dim3(256), 0, st, p);
      launch_timed("route_place", route_place_kernel<false>, dim3(p.chunks), dim3(kPlaceThreads), 0, st, p, log_groups);
    }
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
  auto kernel = p.E <= 64    ? f32 ? route_select_grad_kernel<1, float> : route_select_grad_kernel<1, uint16_t>
                : p.E <= 128 ? f32 ? route_select_grad_kernel<2, float> : route_select_grad_kernel<2, uint16_t>
                             : f32 ? route_select_grad_kernel<4, float> : route_select_grad_kernel<4, uint16_t>;
  launch_timed("route_select_grad", kernel, dim3(min((p.T + 15) / 16, kMaxGrid)), dim3(256), 0, st, p);
  return hipGetLastError();
}

hipError_t launch_pair_positions(const int32_t* order, int m, int n_pairs, int32_t* pos, hipStream_t st) {
  if (n_pairs > 0) launch_timed("pair_fill", pairs_fill_kernel, dim3(grid_of(n_pairs)), dim3(256), 0, st, pos, n_pairs);
  if (m > 0) launch_timed("pair_positions", pairs_invert_kernel, dim3(grid_of(m)), dim3(256), 0, st, order, m, n_pairs, pos);
  return hipGetLastError();
}

}  // namespace mira
