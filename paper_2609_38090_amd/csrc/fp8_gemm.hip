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
#include <type_traits>

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


// ---- many rows: tiles through LDS ---------------------------------------------
//
// A workgroup of WN x WM waves owns BN weight rows by BM token rows; a wave owns
// 16 NT x 16 MT of them, within one scale block of the weights.  Stages of one
// block of the contraction (128 bytes of every row, and their scales) go to LDS
// by direct loads, two stages in turn: the loads of the next one are in flight
// while this one is multiplied.

// One direct-to-LDS load of a wave: lane l's bytes go to LDS address m0 + 16 l
// (or 4 l).  The compiler does not see these loads; every wait for them is the
// explicit one at the stage's start.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma16(const void* src, uint32_t m0) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(src), "s"(m0) : "memory", "m0");
}
__device__ __forceinline__ void dma16(uint32_t off, const void* base, uint32_t m0) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "s"(m0) : "memory", "m0");
}
__device__ __forceinline__ void dma4(const void* src, uint32_t m0) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(src), "s"(m0) : "memory", "m0");
}
#pragma clang diagnostic pop

__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p;
}

// All loads to LDS have landed and all LDS reads have returned, in every wave.
__device__ __forceinline__ void stage_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

struct Tile {
  int g, m0, m1, nt;  // group, rows [m0, m1), tile of weight rows
};

// Tiles are numbered so that the workgroups of one XCD (ids equal modulo 8) take
// consecutive ones, and consecutive tiles run down kTileRun row tiles that share
// their weights before the next weight rows.
constexpr int kTileRun = 8;
__device__ __forceinline__ bool tile_number(int mT, int nT, int& mt, int& nt) {
  const int total = mT * nT, per = (total + 7) >> 3, i = blockIdx.x >> 3;
  const int id = (blockIdx.x & 7) * per + i;
  if (i >= per || id >= total) return false;
  const int run = id / (kTileRun * nT), first = run * kTileRun, rows = min(mT - first, kTileRun);
  const int at = id - first * nT;
  nt = at / rows;
  mt = first + at - nt * rows;
  return true;
}

// The tile of this workgroup, from the groups' row counts; false if there is none.
template <int BM>
__device__ __forceinline__ bool find_tile(const GemmParams& p, int nT, int* shared, Tile& t) {
  if (!p.offsets) {
    int mt;
    if (!tile_number((p.M + BM - 1) / BM, nT, mt, t.nt)) return false;
    t.g = 0;
    t.m0 = mt * BM;
    t.m1 = min(t.m0 + BM, p.M);
    return true;
  }
  if (threadIdx.x < 64) {  // one wave: lane l has groups 4l .. 4l+3
    const int l = threadIdx.x;
    Rows r[4];
    int n[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r[i] = 4 * l + i < p.G ? rows_of(p, 4 * l + i) : Rows{0, 0};
      n[i] = (r[i].hi - r[i].lo + BM - 1) / BM;
      sum += n[i];
    }
    int end = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(end, o, 64);
      if (l >= o) end += v;
    }
    const int mT = __shfl(end, 63, 64);
    int mt = 0, nt = 0;
    const bool any = tile_number(mT, nT, mt, nt);
    if (l == 0) shared[0] = any ? nt : -1;
    int at = end - sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (any && mt >= at && mt < at + n[i]) {
        shared[1] = 4 * l + i;
        shared[2] = r[i].lo + (mt - at) * BM;
        shared[3] = r[i].hi;
      }
      at += n[i];
    }
  }
  __syncthreads();
  t.nt = shared[0];
  t.g = shared[1];
  t.m0 = shared[2];
  t.m1 = min(shared[2] + BM, shared[3]);
  return t.nt >= 0;
}

template <typename OutT>
__device__ __forceinline__ void store_out4(OutT* p, v4f v, int n) {
  if (n >= 4 && ((uintptr_t)p & (4 * sizeof(OutT) - 1)) == 0) {
    if constexpr (sizeof(OutT) == 4) {
      *(v4f*)p = v;
    } else {
      uint16_t h[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) store_out(h + i, v[i]);
      *(uint2*)p = uint2{(uint32_t)h[0] | (uint32_t)h[1] << 16, (uint32_t)h[2] | (uint32_t)h[3] << 16};
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) store_out(p + i, v[i]);
  }
}

// Compile-time loop: f(std::integral_constant<int, I>) for I in [B, E).
template <int B, int E, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (B < E) {
    f(std::integral_constant<int, B>{});
    static_for<B + 1, E>(f);
  }
}

// Operand fragments of one block: as loaded, or widened to bf16.
template <bool EXACT>
struct Frag;
template <>
struct Frag<false> {
  v8i v;
  __device__ __forceinline__ void set(v8i a) { v = a; }
  __device__ __forceinline__ static v4f mul(const Frag& a, const Frag& b) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, v4f{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
  }
};
template <>
struct Frag<true> {
  v4i v[4];
  __device__ __forceinline__ void set(v8i a) {
#pragma unroll
    for (int s = 0; s < 4; ++s) v[s] = widen8(a[2 * s], a[2 * s + 1]);
  }
  __device__ __forceinline__ static v4f mul(const Frag& a, const Frag& b) {
    v4f d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < 4; ++s) d = mfma_bf16(a.v[s], b.v[s], d);
    return d;
  }
};

template <int NT, int MT, int WN, int WM, bool EXACT, typename OutT>
__global__ __launch_bounds__(64 * WN * WM) void fp8_gemm_tile_kernel(GemmParams p, int nT) {
  constexpr int BN = 16 * NT * WN, BM = 16 * MT * WM, W = WN * WM;
  constexpr int kW = BN * 128, kX = BM * 128, kStage = kW + kX, kScales = (BM + 64) * 16;
  constexpr int GW = BN / 8 / W, GX = BM / 8 / W;  // loads of 8 rows per wave and stage
  static_assert(BN % (8 * W) == 0 && BM % (8 * W) == 0 && BM % 64 == 0 && BM / 64 < W && 128 % (16 * NT) == 0, "tile shape");
  __shared__ __attribute__((aligned(1024))) char lds[2 * (kStage + kScales)];
  __shared__ int tile_s[4];
  Tile t;
  if (!find_tile<BM>(p, nT, tile_s, t)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, kg = lane >> 4, wn = wave % WN, wm = wave / WN;
  const int n0 = t.nt * BN;
  const uint8_t* w = p.w + (size_t)t.g * p.w_stride + (size_t)n0 * p.ldw;  // advances with the stages
  const float* ws = p.ws + (size_t)t.g * p.ws_stride;

  // Row r stores its 16-byte chunk c at chunk c ^ ((r >> 1) & 7): a 128-bit read
  // serves rows 0-3 and 12-15 of one k-group with rows 4-11 of the next, and
  // these fall on distinct banks (64 banks, two rows).
  uint32_t gw[GW];  // 32-bit offsets: a tile's weight rows lie within 256 * ldw < 2^32 bytes
  const uint8_t* gx[GX];
  int chunk[2];  // the lane's chunk of even and odd groups of eight rows
#pragma unroll
  for (int j = 0; j < 2; ++j) chunk[j] = (lane & 7) ^ ((4 * j + (lane >> 4)) & 7);
#pragma unroll
  for (int j = 0; j < GW; ++j) {
    const int grp = wave * GW + j;
    const int r = min(grp * 8 + (lane >> 3), p.N - 1 - n0);
    gw[j] = (uint32_t)r * (uint32_t)p.ldw + chunk[grp & 1] * 16;
  }
#pragma unroll
  for (int j = 0; j < GX; ++j) {
    const int grp = wave * GX + j;
    const int src = max(source_row(p, min(t.m0 + grp * 8 + (lane >> 3), t.m1 - 1)), 0);
    gx[j] = p.x + (size_t)src * p.ldx + chunk[grp & 1] * 16;
  }
  // Scales go to LDS for four stages at a time, [row][4] (a load touches a line
  // of memory per row, as many as the rows themselves take): a wave of 64 token
  // rows each, and one for the weights' blocks.  The last four are the last of
  // the row, so that no load passes its end.
  const float* gs = nullptr;
  if (wave < BM / 64)
    gs = p.xs + (size_t)max(source_row(p, min(t.m0 + wave * 64 + lane, t.m1 - 1)), 0) * p.ld_xs;
  else if (wave == BM / 64)
    gs = ws + (size_t)min((n0 >> 7) + (lane & ((BN + 127) / 128 - 1)), (p.N - 1) >> 7) * p.ld_ws;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr(lds));
  const int k16 = (p.K + 15) & ~15;
  // Load d of the wave's GW + GX of a whole stage.
  const auto load_one = [&](auto d, uint32_t at) {
    constexpr int D = d;
    if constexpr (D < GW) {
      dma16(gw[D], w, at + (wave * GW + D) * 1024);
    } else {
      dma16(gx[D - GW], at + kW + (wave * GX + D - GW) * 1024);
      gx[D - GW] += 128;
    }
  };
  const auto load_scales = [&](int q) {  // those of stages 4q .. 4q+3
    const int at = 2 * kStage + (q & 1) * kScales + wave * 1024;
    if (wave > BM / 64 || 4 * q >= p.KB) return;
    if (p.KB >= 4) {
      dma16(gs + min(4 * q, p.KB - 4), lds0 + at);
    } else {
      for (int i = 0; i < p.KB; ++i) *(float*)(lds + at + lane * 16 + i * 4) = gs[i];
    }
  };
  // Any stage at once; where the contraction ends inside it, the chunks behind its end are zeros.
  const auto load_stage = [&](int b) {
    const int buf = (b & 1) * kStage;
    const uint32_t at = lds0 + buf;
    if ((b + 1) * 128 <= k16) {
      static_for<0, GW + GX>([&](auto d) { load_one(d, at); });
    } else {
#pragma unroll
      for (int j = 0; j < GW; ++j) {
        const int grp = wave * GW + j;
        if (b * 128 + chunk[grp & 1] * 16 < k16) dma16(gw[j], w, at + grp * 1024);
        else *(v4i*)(lds + buf + grp * 1024 + lane * 16) = zero16();
      }
#pragma unroll
      for (int j = 0; j < GX; ++j) {
        const int grp = wave * GX + j;
        if (b * 128 + chunk[grp & 1] * 16 < k16) dma16(gx[j], at + kW + grp * 1024);
        else *(v4i*)(lds + buf + kW + grp * 1024 + lane * 16) = zero16();
      }
    }
    w += 128;
  };

  v4f acc[NT][MT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
  const int sw7 = (r16 >> 1) & 7;
  const int o0 = r16 * 128 + (kg ^ sw7) * 16, o1 = r16 * 128 + ((kg + 4) ^ sw7) * 16;
  const auto read = [&](const char* base) { return join(*(const v4i*)(base + o0), *(const v4i*)(base + o1)); };

  // Multiplies stage b.  Step i * MT + j multiplies weight tile i by token tile j
  // and adds the sums of kBehind steps before, so that neither the matrix core
  // nor the fp32 additions wait for one another; the fences keep this order.
  // LOAD: the loads of stage b + 1, a whole one, are issued between the steps.
  constexpr int kSteps = NT * MT, kBehind = EXACT ? 1 : 2, kLoads = GW + GX;
  const auto multiply = [&](int b, auto load) {
    constexpr bool LOAD = load;
    const char* st = lds + (b & 1) * kStage;
    const uint32_t next = lds0 + ((b + 1) & 1) * kStage;
    const char* sx = st + kW + wm * (MT * 2048);
    const char* sw = st + wn * (NT * 2048);
    const int q = b >> 2;
    const float* sc = (const float*)(lds + 2 * kStage + (q & 1) * kScales) + (b - max(min(4 * q, p.KB - 4), 0));
    v4f d[kBehind + 1];
    Frag<EXACT> a[2], x[MT];
    float s[MT];
    v8i raw = read(sw);
    v8i xr[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) xr[j] = read(sx + j * 2048);
    const float wsc = sc[(BM + (wn * NT) / 8) * 4];
#pragma unroll
    for (int j = 0; j < MT; ++j) s[j] = sc[(wm * (MT * 16) + j * 16 + r16) * 4];
    a[0].set(raw);
    static_for<0, kSteps + kBehind>([&](auto step) {
      constexpr int S = step, i = S / MT, j = S % MT;
      if constexpr (S < kSteps) {
        if constexpr (i == 0) {
          x[j].set(xr[j]);
          s[j] *= wsc;
        }
        if constexpr (j == 0 && i + 1 < NT) raw = read(sw + (i + 1) * 2048);
        d[S % (kBehind + 1)] = Frag<EXACT>::mul(a[i & 1], x[j]);
        if constexpr (j == MT - 1 && i + 1 < NT) a[(i + 1) & 1].set(raw);
      }
      if constexpr (S >= kBehind) {
        constexpr int P = S - kBehind;
        v4f& c = acc[P / MT][P % MT];
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = fmaf(d[P % (kBehind + 1)][e], s[P % MT], c[e]);
      }
      if constexpr (LOAD && S >= 1 && S <= kLoads) load_one(std::integral_constant<int, S - 1>{}, next);
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (LOAD) w += 128;
  };
  const int whole = k16 >> 7;
  load_scales(0);
  load_stage(0);
  int b = 0;
  for (; b + 1 < whole; ++b) {
    stage_barrier();
    if ((b & 3) == 1) load_scales((b >> 2) + 1);
    multiply(b, std::true_type{});
  }
  for (; b < p.KB; ++b) {
    stage_barrier();
    if ((b & 3) == 1) load_scales((b >> 2) + 1);
    if (b + 1 < p.KB) load_stage(b + 1);
    multiply(b, std::false_type{});
  }

  OutT* out = (OutT*)p.out;
#pragma unroll
  for (int j = 0; j < MT; ++j) {
    const int m = t.m0 + wm * (MT * 16) + j * 16 + r16;
    if (m >= t.m1) continue;
    const bool none = p.order && source_row(p, m) < 0;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int n = n0 + wn * (NT * 16) + i * 16 + 4 * kg;
      if (n < p.N) store_out4(out + (size_t)m * p.ldo + n, none ? v4f{0.f, 0.f, 0.f, 0.f} : acc[i][j], p.N - n);
    }
  }
}

template <int NT, int MT, int WN, int WM, bool EXACT, typename OutT>
void launch_tile(const GemmParams& p, hipStream_t st) {
  constexpr int BN = 16 * NT * WN, BM = 16 * MT * WM;
  const int nT = (p.N + BN - 1) / BN;
  // an upper bound of the row tiles: every group may end inside one
  const long mT = p.offsets ? p.M / BM + (p.G < p.M ? p.G : p.M) : (p.M + BM - 1) / BM;
  const long grid = (mT * nT + 7) / 8 * 8;
  launch_timed("fp8_gemm_tile", fp8_gemm_tile_kernel<NT, MT, WN, WM, EXACT, OutT>, dim3((uint32_t)grid),
               dim3(64 * WN * WM), 0, st, p, nT);
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
  if (p.M > 16 * p.G) {
    if (a.out_dtype == MIRA_F32) launch_tile<8, 4, 2, 4, true, float>(p, st);
    else launch_tile<8, 4, 2, 4, false, uint16_t>(p, st);
    return hipGetLastError();
  }
  const dim3 grid((p.N + 15) / 16, p.G);
  if (a.out_dtype == MIRA_F32)
    launch_timed("fp8_gemm_rows", fp8_gemm_rows_kernel<float>, grid, dim3(256), 0, st, p);
  else
    launch_timed("fp8_gemm_rows", fp8_gemm_rows_kernel<uint16_t>, grid, dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace mira
