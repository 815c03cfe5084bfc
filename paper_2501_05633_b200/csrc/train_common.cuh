// What the training operators share: element types, the dropout generator, warp sums, host-side checks.
#ifndef REGTOPK_TRAIN_COMMON_CUH_
#define REGTOPK_TRAIN_COMMON_CUH_

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "regtopk_train.h"

namespace {

typedef uint32_t u32;

constexpr u32 kAll = 0xFFFFFFFFu;

// ---- element types ---------------------------------------------------------------------------------------------
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// Eight consecutive elements as they lie in memory: one 16-byte word of a 16-bit type, two of binary32.
template <typename T> struct Eight {
  static constexpr int kWords = sizeof(T) / 2;
  uint4 w[kWords];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < kWords; ++i) reinterpret_cast<uint4*>(p)[i] = w[i];
  }
  __device__ __forceinline__ float get(int j) const { return to_float(reinterpret_cast<const T*>(w)[j]); }
  __device__ __forceinline__ void set(int j, float v) { reinterpret_cast<T*>(w)[j] = from_float<T>(v); }
};

// ---- dropout ---------------------------------------------------------------------------------------------------
struct Drop {
  u32 threshold;  // an element is kept if its 16-bit number is at least this; 0: no dropout
  float scale;
  u32 key0, key1, subsequence;
};

// Keep bits of the eight columns 8*group .. 8*group + 7 of a row, bit j for column 8*group + j: one call of
// Philox4x32-10 gives them all.  Sixteen bits a column, not thirty-two: p is a multiple of 2^-16 then, and the
// generator costs half (ten rounds are 20 multiplies and 20 three-input exclusive-ors for eight columns).
__device__ __forceinline__ u32 keep_bits(const Drop& d, uint64_t row, u32 group) {
  u32 c0 = group, c1 = (u32)row, c2 = (u32)(row >> 32), c3 = d.subsequence, k0 = d.key0, k1 = d.key1;
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (u32)(b >> 32) ^ c1 ^ k0;
    c1 = (u32)b;
    c2 = (u32)(a >> 32) ^ c3 ^ k1;
    c3 = (u32)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  const u32 w[4] = {c0, c1, c2, c3};
  u32 bits = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) bits |= (((j & 1) ? w[j >> 1] >> 16 : w[j >> 1] & 0xFFFFu) >= d.threshold ? 1u : 0u) << j;
  return bits;
}

// ---- a row's columns over the lanes of a warp --------------------------------------------------------------------
// A warp holds a row in units of 256 columns, eight of them per lane: eight neighbours where rows are 16-byte aligned
// (VEC, one wide access), otherwise every 32nd column (eight narrow accesses that are each contiguous over the warp).
template <bool VEC> __device__ __forceinline__ int lane_col(int lane, int j) { return VEC ? lane * 8 + j : j * 32 + lane; }

// The keep bits of this lane's eight columns of the unit that begins at column `col0` (a multiple of 256).
template <bool VEC> __device__ __forceinline__ u32 unit_keep_bits(const Drop& d, uint64_t row, int64_t col0, int lane) {
  const u32 own = keep_bits(d, row, (u32)(col0 >> 3) + lane);
  if (VEC) return own;
  u32 bits = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j)  // column j*32 + lane belongs to the group that lane j*4 + lane/8 has drawn
    bits |= ((__shfl_sync(kAll, own, j * 4 + (lane >> 3)) >> (lane & 7)) & 1u) << j;
  return bits;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}

// ---- host --------------------------------------------------------------------------------------------------------
inline int train_rc(cudaError_t e) {
  if (e == cudaSuccess) return REGTOPK_OK;
  cudaGetLastError();
  return e == cudaErrorNoDevice || e == cudaErrorInsufficientDriver || e == cudaErrorNoKernelImageForDevice
             ? REGTOPK_ERR_NO_DEVICE : REGTOPK_ERR_CUDA;
}

constexpr int kMaxDevices = 64;

// The current device and its SM count (looked up once per device); false without a usable one.
inline bool current_device(int* dev, int* sms) {
  static int known[kMaxDevices];
  if (cudaGetDevice(dev) != cudaSuccess || *dev < 0 || *dev >= kMaxDevices) { cudaGetLastError(); return false; }
  int n = __atomic_load_n(&known[*dev], __ATOMIC_RELAXED);
  if (!n) {
    int major = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, *dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, *dev) != cudaSuccess || major != 10) {
      cudaGetLastError();
      return false;
    }
    __atomic_store_n(&known[*dev], n, __ATOMIC_RELAXED);
  }
  *sms = n;
  return true;
}

inline bool make_drop(const regtopk_dropout_params* p, Drop* d) {
  d->threshold = 0;
  d->scale = 1.0f;
  d->key0 = d->key1 = d->subsequence = 0;
  if (!p) return true;
  if (!(p->p >= 0.0 && p->p <= 1.0)) return false;
  d->threshold = (u32)rint(65536.0 * p->p);
  d->scale = d->threshold < 65536u ? (float)(65536.0 / (65536.0 - d->threshold)) : 0.0f;
  d->key0 = (u32)p->seed;
  d->key1 = (u32)(p->seed >> 32);
  d->subsequence = p->subsequence;
  return true;
}

inline size_t type_size(int32_t t) { return t == REGTOPK_TYPE_F32 ? 4 : t == REGTOPK_TYPE_BF16 || t == REGTOPK_TYPE_F16 ? 2 : 0; }

// Whether every row of the matrix begins on a 16-byte boundary (NULL: nothing to read).
inline bool rows_aligned(const void* p, int64_t ld, size_t size, int64_t rows) {
  return !p || ((uintptr_t)p % 16 == 0 && (rows <= 1 || (uint64_t)ld * size % 16 == 0));
}

inline bool good_matrix(const void* p, int64_t ld, int64_t rows, int64_t cols, size_t size) {
  return p && (uintptr_t)p % size == 0 && (rows <= 1 || ld >= cols);
}

}  // namespace
#endif
