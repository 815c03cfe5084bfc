// 8-bit rows (include/regtopk_experts.h): blocks of 32 columns of e4m3 numbers that share a power of two.
#ifndef REGTOPK_ROWS8_CUH_
#define REGTOPK_ROWS8_CUH_

#include <cuda_fp8.h>

#include "norm_rows.cuh"
#include "regtopk_experts.h"

namespace {

constexpr u32 kInfinity = 0x7F800000u;  // binary32's, without its sign; above it are the NaN

// The scale byte of a block whose largest finite magnitude has these bits.  448 = 1.75 * 2^8, so that of a value 1.m * 2^(E-127)
// the exponent E - 8 is enough if 1.m <= 1.75, and one more otherwise.
__device__ __forceinline__ u32 scale_byte(u32 most) {
  const int b = (int)(most >> 23) - 8 + ((most & 0x7FFFFFu) > 0x600000u);
  return b > 0 ? (u32)b : 0u;
}
__device__ __forceinline__ float inverse_scale(u32 byte) { return __uint_as_float((254u - byte) << 23); }  // of one that scale_byte gives
__device__ __forceinline__ float scale_value(u32 byte) {
  return __uint_as_float(byte == 0 ? 0x400000u : byte == 255u ? 0x7FC00000u : byte << 23);
}

__device__ __forceinline__ u32 magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ __forceinline__ u32 finite_magnitude(float v) { return magnitude(v) < kInfinity ? magnitude(v) : 0u; }
__device__ __forceinline__ float without_infinity(float v) { return magnitude(v) < kInfinity ? v : __uint_as_float(0x7FC00000u); }
__device__ __forceinline__ u32 e4m3_pair(float a, float b) {
  return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float2 pair_value(u32 pair) {
  return __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)pair, __NV_E4M3)));
}

// Eight neighbours, a thread's, to their place in an 8-bit row (at values, with their block's scale at *scale).  Four threads in a row share
// a block and the whole warp takes part; `there`: the columns exist, otherwise f holds zeros.
__device__ __forceinline__ void store_rows8(const Octet& given, uint8_t* values, uint8_t* scale, bool there) {
  Octet f;
  float top = 0.0f;  // NaN are passed over
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[i] = given[i];
    top = fmaxf(top, fmaxf(fabsf(f[i].x), fabsf(f[i].y)));
  }
  u32 most = __float_as_uint(top);
  most = max(most, __shfl_xor_sync(kAll, most, 1));
  most = max(most, __shfl_xor_sync(kAll, most, 2));
  if (__any_sync(kAll, most >= kInfinity)) {
    most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      most = max(most, max(finite_magnitude(f[i].x), finite_magnitude(f[i].y)));
      f[i] = make_float2(without_infinity(f[i].x), without_infinity(f[i].y));
    }
    most = max(most, __shfl_xor_sync(kAll, most, 1));
    most = max(most, __shfl_xor_sync(kAll, most, 2));
  }
  const u32 byte = scale_byte(most);
  const float2 inverse = both(inverse_scale(byte));
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = mul2(f[i], inverse);
  if (!there) return;
  uint2 v;
  v.x = e4m3_pair(f[0].x, f[0].y) | e4m3_pair(f[1].x, f[1].y) << 16;
  v.y = e4m3_pair(f[2].x, f[2].y) | e4m3_pair(f[3].x, f[3].y) << 16;
  *reinterpret_cast<uint2*>(values) = v;
  if (!(threadIdx.x & 3)) *scale = (uint8_t)byte;
}

// A warp's 256 columns of a row from one that is a multiple of 256 on, every 32nd a lane's: element j is column j * 32 + lane.  `at` is
// the lane's first, `left` how many columns there are from it on; WHOLE: all 256 are there, which spares a comparison for each.  Past
// the end f holds zeros.
template <typename T, bool WHOLE> __device__ __forceinline__ void read_apart(Octet& f, const T* at, int left) {
  T v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = WHOLE || j * 32 < left ? at[j * 32] : from_float<T>(0.0f);
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = make_float2(to_float(v[2 * i]), to_float(v[2 * i + 1]));
}
template <typename T, bool WHOLE> __device__ __forceinline__ void store_apart(const Octet& f, T* at, int left) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (WHOLE || j * 32 < left) at[j * 32] = from_float<T>((j & 1) ? f[j >> 1].y : f[j >> 1].x);
}
// The same of an 8-bit row; `scales`: of the first of the 256 columns.  The whole warp takes part.
template <bool WHOLE> __device__ __forceinline__ void store_rows8_apart(const Octet& f, uint8_t* at, uint8_t* scales, int lane, int left) {
  u32 own = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float e[2] = {f[i].x, f[i].y};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      u32 most = __reduce_max_sync(kAll, magnitude(e[j]));
      if (most >= kInfinity) {
        most = __reduce_max_sync(kAll, finite_magnitude(e[j]));
        e[j] = without_infinity(e[j]);
      }
      const u32 byte = scale_byte(most);
      e[j] *= inverse_scale(byte);
      own = lane == 2 * i + j ? byte : own;
    }
    const u32 pair = e4m3_pair(e[0], e[1]);
    if (WHOLE || i * 64 < left) at[i * 64] = (uint8_t)pair;
    if (WHOLE || i * 64 + 32 < left) at[i * 64 + 32] = (uint8_t)(pair >> 8);
  }
  if (lane < 8 && (WHOLE || lane * 31 < left)) scales[lane] = (uint8_t)own;  // lane * 32 < left + lane
}
template <bool WHOLE> __device__ __forceinline__ void read_rows8_apart(Octet& f, const uint8_t* at, const uint8_t* scales, int lane, int left) {
  const float own = scale_value(lane < 8 && (WHOLE || lane * 31 < left) ? scales[lane] : 0u);
  u32 v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = WHOLE || j * 32 < left ? at[j * 32] : 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    f[i] = mul2(pair_value(v[2 * i] | v[2 * i + 1] << 8), make_float2(__shfl_sync(kAll, own, 2 * i), __shfl_sync(kAll, own, 2 * i + 1)));
}

// Eight neighbours of an 8-bit row, as they lie in memory.
struct Packed8 {
  uint2 v;
  u32 byte;
  __device__ __forceinline__ void fetch(const uint8_t* values, const uint8_t* scale) {
    v = *reinterpret_cast<const uint2*>(values);
    byte = *scale;
  }
  __device__ __forceinline__ void clear() { v = make_uint2(0, 0), byte = 0; }
  __device__ __forceinline__ void get(Octet& f) const {
    const float2 scale = both(scale_value(byte));
    f[0] = mul2(pair_value(v.x & 0xFFFFu), scale);
    f[1] = mul2(pair_value(v.x >> 16), scale);
    f[2] = mul2(pair_value(v.y & 0xFFFFu), scale);
    f[3] = mul2(pair_value(v.y >> 16), scale);
  }
};

inline int64_t blocks_of(int64_t cols) { return (cols + 31) / 32; }
inline bool good_rows8(const uint8_t* values, int64_t ld_values, const uint8_t* scales, int64_t ld_scales, int64_t rows, int64_t cols, int halves) {
  return values && scales && (rows <= 1 || (ld_values >= halves * cols && ld_scales >= halves * blocks_of(cols)));
}
inline bool rows8_aligned(const uint8_t* values, int64_t ld, int64_t rows) { return !values || ((uintptr_t)values % 8 == 0 && (rows <= 1 || ld % 8 == 0)); }

// ---- rows and columns of a flat index -----------------------------------------------------------------------------
// n / d for n < 2^31 by a multiplication (Granlund and Montgomery 1994): with 2^(s-1) < d <= 2^s and magic =
// floor(2^(31+s) / d) + 1, which has 32 bits, floor(n / d) = floor(2n magic / 2^(32+s)).
struct Divisor {
  u32 d, magic, shift;
  __device__ __forceinline__ u32 quotient_of(u32 n) const { return __umulhi(2 * n, magic) >> shift; }
};
inline Divisor divisor(int64_t d) {
  int s = 0;
  while (((int64_t)1 << s) < d) ++s;
  return {(u32)d, (u32)(((uint64_t)1 << (31 + s)) / (uint64_t)d + 1), (u32)s};
}

}  // namespace
#endif
