// Rows of any length and alignment and their e4m3 form, for the kernels that walk
// rows eight columns to a lane (16 lanes hold a block of 128 that shares a scale).
#pragma once

#include "device_util.h"
#include "mira_internal.h"

namespace mira {

constexpr float kE4m3Max = 448.f;

// Four values to four e4m3 bytes (nearest even; |v| <= 448 (1 + 2^-23), which rounds to 448).
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}

__device__ __forceinline__ float max_abs(float m, float v) { return fmaxf(m, fabsf(v)); }

// Maximum over each 16 consecutive lanes, in all of them.
__device__ __forceinline__ float max16(float v) {
  v = fmaxf(v, dpp<0xB1>(v));
  v = fmaxf(v, dpp<0x4E>(v));
  v = fmaxf(v, dpp<0x141>(v));
  return fmaxf(v, dpp<0x140>(v));
}

// Vectors at the alignment of their elements: global loads take any, so rows of
// every length and start load 16 bytes at a time.
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));
typedef int v4i_any __attribute__((ext_vector_type(4), aligned(2)));
typedef int v2i_any __attribute__((ext_vector_type(2), aligned(2)));

__device__ __forceinline__ void load_n(const float* p, float (&v)[4]) {
  const v4f q = *(const v4f_any*)p;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = q[i];
}
__device__ __forceinline__ void load_n(const uint16_t* p, float (&v)[4]) {
  const v2i_any q = *(const v2i_any*)p;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    v[2 * i] = __uint_as_float((uint32_t)q[i] << 16);
    v[2 * i + 1] = __uint_as_float((uint32_t)q[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load_n(const float* p, float (&v)[8]) {
  const v4f a = *(const v4f_any*)p, b = *(const v4f_any*)(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = a[i];
    v[4 + i] = b[i];
  }
}
__device__ __forceinline__ void load_n(const uint16_t* p, float (&v)[8]) {
  const v4i q = *(const v4i_any*)p;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float((uint32_t)q[i] << 16);
    v[2 * i + 1] = __uint_as_float((uint32_t)q[i] & 0xFFFF0000u);
  }
}

// N values of a row from column c on; those from cols on are 0.
template <int N, typename T>
__device__ __forceinline__ void load_cols(const T* row, int c, int cols, float (&v)[N]) {
  if (c + N <= cols) {
    load_n(row + c, v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = c + i < cols ? load_act(row, c + i) : 0.f;
  }
}

// Eight values of a row as they were loaded, widened where they are used: half the
// registers for bf16.
template <typename T>
struct Raw8;
template <>
struct Raw8<float> {
  v4f a, b;
  __device__ __forceinline__ float operator[](int i) const { return i < 4 ? a[i] : b[i - 4]; }
  __device__ __forceinline__ void load(const float* p) {
    a = *(const v4f_any*)p;
    b = *(const v4f_any*)(p + 4);
  }
  __device__ __forceinline__ void zero() { a = b = v4f{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void put(int i, float v) {
    if (i < 4) a[i] = v;
    else b[i - 4] = v;
  }
  // n values move out in front, zeros in behind.
  __device__ __forceinline__ void shift(int n) {
    if (n & 4) a = b, b = v4f{0.f, 0.f, 0.f, 0.f};
    if (n & 2) a = v4f{a[2], a[3], b[0], b[1]}, b = v4f{b[2], b[3], 0.f, 0.f};
    if (n & 1) a = v4f{a[1], a[2], a[3], b[0]}, b = v4f{b[1], b[2], b[3], 0.f};
    if (n >= 8) zero();
  }
};
template <>
struct Raw8<uint16_t> {
  v4i q;
  __device__ __forceinline__ float operator[](int i) const {
    const uint32_t u = (uint32_t)q[i >> 1];
    return __uint_as_float(i & 1 ? u & 0xFFFF0000u : u << 16);
  }
  __device__ __forceinline__ void load(const uint16_t* p) { q = *(const v4i_any*)p; }
  __device__ __forceinline__ void zero() { q = v4i{0, 0, 0, 0}; }
  __device__ __forceinline__ void put(int i, uint16_t v) { q[i >> 1] |= (int)((uint32_t)v << (i & 1 ? 16 : 0)); }
  __device__ __forceinline__ void shift(int n) {
    if (n & 4) q = v4i{q[2], q[3], 0, 0};
    if (n & 2) q = v4i{q[1], q[2], q[3], 0};
    if (n & 1) {
      auto half = [](int lo, int hi) { return (int)((uint32_t)lo >> 16 | (uint32_t)hi << 16); };
      q = v4i{half(q[0], q[1]), half(q[1], q[2]), half(q[2], q[3]), half(q[3], 0)};
    }
    if (n >= 8) zero();
  }
};
// Columns c .. c + 7 of a row.  A lane at the row's end loads the row's last eight, and settle(), called
// once all loads are on their way, moves them to their places, zeros behind: a load behind a
// condition of its own would be waited for before the next (a row's three loads one after another:
// 30000 x 700 bf16 82 us for a norm's gradient, 42 so).
template <typename T>
__device__ __forceinline__ void load_raw(const T* row, int c, int cols, Raw8<T>& v) {
  if (cols >= 8) {  // (the same for all)
    v.load(row + min(c, cols - 8));
  } else {
    v.zero();
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < cols) v.put(i, row[c + i]);
  }
}
template <typename T>
__device__ __forceinline__ void settle(Raw8<T>& v, int c, int cols) {
  if (cols >= 8 && c + 8 > cols) v.shift(c + 8 - cols);
}

// Two values to two bf16, nearest even, NaN kept (one instruction on gfx950).
__device__ __forceinline__ uint32_t to_bf16x2(float a, float b) {
  typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
  const v2bf r = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ uint16_t to_bf16(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }

__device__ __forceinline__ void store_act(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_act(uint16_t* p, float v) { *p = to_bf16(v); }

// Eight values of a row from column c on, those before cols.
__device__ __forceinline__ void store8(float* p, const float v[8]) {
  *(v4f_any*)p = v4f{v[0], v[1], v[2], v[3]};
  *(v4f_any*)(p + 4) = v4f{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void store8(uint16_t* p, const float v[8]) {
  *(v4i_any*)p = v4i{(int)to_bf16x2(v[0], v[1]), (int)to_bf16x2(v[2], v[3]), (int)to_bf16x2(v[4], v[5]),
                     (int)to_bf16x2(v[6], v[7])};
}
template <typename T>
__device__ __forceinline__ void store_cols(T* row, int c, int cols, const float v[8]) {
  if (c + 8 <= cols) {
    store8(row + c, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < cols) store_act(row + c + i, v[i]);
  }
}

// Values as a row of T holds them.
__device__ __forceinline__ float held(float v, const float*) { return v; }
__device__ __forceinline__ float held(float v, const uint16_t*) { return bf16_to_f32(to_bf16(v)); }

__device__ __forceinline__ float max_abs8(const float v[8]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max_abs(m, v[i]);
  return m;
}

// A lane's eight values as e4m3: inv is its block's 448 / maximum.
__device__ __forceinline__ uint2 to_e4m3x8(const float v[8], float inv) {
  return uint2{to_e4m3(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
               to_e4m3(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv)};
}

// Zeros in place of what is beyond a row's columns (a factor may have made -0 or NaN of it).
__device__ __forceinline__ void clear_beyond(float (&v)[8], int c, int cols) {
  if (c + 8 > cols) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? v[i] : 0.f;
  }
}
// A row's block of maximum m: 16 lanes, eight columns each from c on (zeros beyond the row), write the
// row's bytes up to the next multiple of 16 columns and the block's scale.
__device__ __forceinline__ void store_block(const float (&v)[8], float m, int c, int cols, uint8_t* q, float* scale) {
  if (c >= (int)align_up((size_t)cols, 16)) return;
  if ((c & 127) == 0) scale[c >> 7] = m / kE4m3Max;
  *(uint2*)(q + c) = to_e4m3x8(v, kE4m3Max / m);
}
// ... whose maximum is to be found.
__device__ __forceinline__ void quantize_block(float (&v)[8], int c, int cols, float eps, uint8_t* q, float* scale) {
  clear_beyond(v, c, cols);
  store_block(v, fmaxf(max16(max_abs8(v)), eps), c, cols, q, scale);
}

}  // namespace mira
