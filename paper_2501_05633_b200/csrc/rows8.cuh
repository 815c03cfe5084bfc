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

// Eight of a lane's values, laid out as read_eight does, to their place in the 8-bit row; columns from `cols` on are zeros in f and
// not written.  The whole warp takes part; VEC: four lanes in a row, whose first one's column is a multiple of 32, share a block.
template <bool VEC> __device__ __forceinline__ void store_rows8(const Octet& given, uint8_t* values, uint8_t* scales, int64_t c0, int lane, int64_t cols) {
  Octet f;
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = given[i];
  if (VEC) {
    u32 most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) most = max(most, max(magnitude(f[i].x), magnitude(f[i].y)));
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
    const int64_t c = c0 + lane * 8;
    if (c < cols) {
      uint2 v;
      v.x = e4m3_pair(f[0].x, f[0].y) | e4m3_pair(f[1].x, f[1].y) << 16;
      v.y = e4m3_pair(f[2].x, f[2].y) | e4m3_pair(f[3].x, f[3].y) << 16;
      *reinterpret_cast<uint2*>(values + c) = v;
      if (!(c & 31)) scales[c >> 5] = (uint8_t)byte;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float v = (j & 1) ? f[j >> 1].y : f[j >> 1].x;
      u32 most = __reduce_max_sync(kAll, magnitude(v));
      if (most >= kInfinity) {
        most = __reduce_max_sync(kAll, finite_magnitude(v));
        v = without_infinity(v);
      }
      const u32 byte = scale_byte(most);
      const int64_t c = c0 + j * 32 + lane;
      if (c < cols) {
        values[c] = (uint8_t)e4m3_pair(v * inverse_scale(byte), 0.0f);
        if (lane == 0) scales[c >> 5] = (uint8_t)byte;
      }
    }
  }
}

// The same eight columns of an 8-bit row; zeros from `cols` on.
template <bool VEC> __device__ __forceinline__ void read_rows8(Octet& f, const uint8_t* values, const uint8_t* scales, int64_t c0, int lane, int64_t cols) {
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = both(0.0f);
  if (VEC) {
    const int64_t c = c0 + lane * 8;
    if (c >= cols) return;
    const uint2 v = *reinterpret_cast<const uint2*>(values + c);
    const float2 scale = both(scale_value(scales[c >> 5]));
    f[0] = mul2(pair_value(v.x & 0xFFFFu), scale);
    f[1] = mul2(pair_value(v.x >> 16), scale);
    f[2] = mul2(pair_value(v.y & 0xFFFFu), scale);
    f[3] = mul2(pair_value(v.y >> 16), scale);
  } else {
    float e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t c = c0 + j * 32 + lane;
      e[j] = c < cols ? pair_value(values[c]).x * scale_value(scales[c >> 5]) : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(e[2 * i], e[2 * i + 1]);
  }
}

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
