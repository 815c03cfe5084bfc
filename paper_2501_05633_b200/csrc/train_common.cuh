// What the training operators share: element types, the dropout generator, warp sums, host-side checks.
#ifndef REGTOPK_TRAIN_COMMON_CUH_
#define REGTOPK_TRAIN_COMMON_CUH_

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include "regtopk_train.h"

namespace {

typedef uint32_t u32;

constexpr u32 kAll = 0xFFFFFFFFu;

// ---- element types ---------------------------------------------------------------------------------------------
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
__device__ __forceinline__ u32 packed(float a, float b, __nv_bfloat16) {  // two rounded values as they lie in memory
  const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const u32*>(&p);
}
__device__ __forceinline__ u32 packed(float a, float b, __half) {
  const __half2 p = __floats2half2_rn(a, b);
  return *reinterpret_cast<const u32*>(&p);
}
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// Arithmetic on two binary32 values in one instruction (both halves rounded as the single ones are).
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n.reg .b64 p, q, r;\nmov.b64 p, {%2, %3};\nmov.b64 q, {%4, %5};\nadd.rn.f32x2 r, p, q;\nmov.b64 {%0, %1}, r;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n.reg .b64 p, q, r;\nmov.b64 p, {%2, %3};\nmov.b64 q, {%4, %5};\nmul.rn.f32x2 r, p, q;\nmov.b64 {%0, %1}, r;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n.reg .b64 p, q, r, s;\nmov.b64 p, {%2, %3};\nmov.b64 q, {%4, %5};\nmov.b64 r, {%6, %7};\nfma.rn.f32x2 s, p, q, r;\nmov.b64 {%0, %1}, s;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// 2^x and 1 / x by the hardware, 2 and 1 units in the last place off, without care for the smallest numbers.
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float reciprocal_fast(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float kLog2E = 1.4426950408889634f;

// Eight elements are held as four pairs: element j is half j % 2 of pair j / 2.
typedef float2 Octet[4];

// Eight consecutive elements as they lie in memory: one 16-byte word of a 16-bit type, two of binary32.
template <typename T> struct Eight {
  static constexpr int kWords = sizeof(T) / 2;
  uint4 w[kWords];
  __device__ __forceinline__ void load(const T* p) {  // shared memory
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  // Global memory.  Eight binary32 values go as one 32-byte access: in two of 16 bytes a warp would touch every 32-byte
  // sector twice.
  __device__ __forceinline__ void fetch(const T* p) {
    if constexpr (kWords == 2)
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(w[0].x), "=r"(w[0].y), "=r"(w[0].z), "=r"(w[0].w), "=r"(w[1].x), "=r"(w[1].y), "=r"(w[1].z), "=r"(w[1].w) : "l"(p));
    else
      w[0] = *reinterpret_cast<const uint4*>(p);
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (kWords == 2)
      asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                   ::"r"(w[0].x), "r"(w[0].y), "r"(w[0].z), "r"(w[0].w), "r"(w[1].x), "r"(w[1].y), "r"(w[1].z), "r"(w[1].w), "l"(p) : "memory");
    else
      *reinterpret_cast<uint4*>(p) = w[0];
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void get(Octet& f) const {
    const T* e = reinterpret_cast<const T*>(w);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(to_float(e[2 * i]), to_float(e[2 * i + 1]));
  }
  __device__ __forceinline__ void put(const Octet& f) {  // rounds all eight
    u32* o = reinterpret_cast<u32*>(w);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) {
        o[i] = packed(f[i].x, f[i].y, T());
      } else {
        o[2 * i] = __float_as_uint(f[i].x);
        o[2 * i + 1] = __float_as_uint(f[i].y);
      }
    }
  }
};

// ---- dropout ---------------------------------------------------------------------------------------------------
struct Drop {
  u32 threshold;  // an element is kept if its 16-bit number is at least this; 0: no dropout, 65536: nothing is kept
  float scale;
  u32 subsequence;
  u32 keys[20];  // the two words of the key of each round
};

// The numbers of eight neighbouring columns, two in a word: one call of Philox4x32-10 gives them all.  Sixteen bits a
// column, not thirty-two: p is a multiple of 2^-16 then, and the generator costs half (ten rounds are 20 multiplies and 20
// three-input exclusive-ors for eight columns; the rounds' keys are constants of the launch).
struct Numbers {
  u32 w[4];
  __device__ __forceinline__ Numbers(const Drop& d, uint64_t row, u32 group) {
    u32 c0 = group, c1 = (u32)row, c2 = (u32)(row >> 32), c3 = d.subsequence;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
      c0 = (u32)(b >> 32) ^ c1 ^ d.keys[2 * i];
      c1 = (u32)b;
      c2 = (u32)(a >> 32) ^ c3 ^ d.keys[2 * i + 1];
      c3 = (u32)a;
    }
    w[0] = c0; w[1] = c1; w[2] = c2; w[3] = c3;
  }
  // Compared in the upper half of a word, where the threshold is too (65536 does not fit there and is tested on its own).
  __device__ __forceinline__ bool keeps(int j, const Drop& d) const {
    return ((j & 1) ? w[j >> 1] : w[j >> 1] << 16) >= d.threshold << 16 && d.threshold < 65536u;
  }
  __device__ __forceinline__ void drop(Octet& f, const Drop& d) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] = mul2(f[i], both(d.scale));
      f[i] = make_float2(keeps(2 * i, d) ? f[i].x : 0.0f, keeps(2 * i + 1, d) ? f[i].y : 0.0f);
    }
  }
};

// ---- a row's columns over the lanes of a warp --------------------------------------------------------------------
// A warp holds a row in units of 256 columns, eight of them per lane: eight neighbours where rows are 16-byte aligned
// (VEC, one wide access), otherwise every 32nd column (eight narrow accesses that are each contiguous over the warp).
template <bool VEC> __device__ __forceinline__ int lane_col(int lane, int j) { return VEC ? lane * 8 + j : j * 32 + lane; }

// Dropout of this lane's eight columns of the unit that begins at column `col0`, a multiple of 256.
template <bool VEC> __device__ __forceinline__ void drop_unit(Octet& f, const Drop& d, uint64_t row, int64_t col0, int lane) {
  const Numbers n(d, row, (u32)(col0 >> 3) + lane);
  if (VEC) {
    n.drop(f, d);
    return;
  }
  u32 own = 0, bits = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) own |= (u32)n.keeps(j, d) << j;
#pragma unroll
  for (int j = 0; j < 8; ++j)  // column j*32 + lane belongs to the group that lane j*4 + lane/8 has drawn
    bits |= ((__shfl_sync(kAll, own, j * 4 + (lane >> 3)) >> (lane & 7)) & 1u) << j;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    f[i] = make_float2((bits >> 2 * i) & 1u ? f[i].x * d.scale : 0.0f, (bits >> (2 * i + 1)) & 1u ? f[i].y * d.scale : 0.0f);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}

// ---- barriers in shared memory for asynchronous copies -----------------------------------------------------------
__device__ __forceinline__ u32 smem_at(const void* p) { return (u32)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(u32 bar, u32 count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count)); }
__device__ __forceinline__ void bar_expect(u32 bar, u32 bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(u32 bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool bar_done(u32 bar, u32 parity) {
  u32 ok;
  asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok;
}

// Every wait ends: after four billion cycles (two seconds at the highest clock) the block gives up, says so here, and leaves
// (regtopk_train_status).
__device__ unsigned int g_gave_up;
constexpr long long kPatience = 4000000000ll;

__device__ __noinline__ bool bar_wait_long(u32 bar, u32 parity, volatile u32* quit) {
  long long began = 0;
  for (u32 tries = 1; !bar_done(bar, parity); ++tries) {
    if (tries % 32) continue;
    const long long now = clock64();
    if (!began) began = now;
    if (*quit) return false;
    if (now - began > kPatience) {
      *quit = 1;
      atomicExch(&g_gave_up, 1u);
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ bool bar_wait(u32 bar, u32 parity, volatile u32* quit) {
  return bar_done(bar, parity) || bar_wait_long(bar, parity, quit);
}

// ---- launches that overlap ---------------------------------------------------------------------------------------
// Every kernel here is launched with programmatic stream serialisation: its blocks may be started while the kernel before
// it in the stream still runs.  It lets its own successor start early in turn, and waits for its predecessor before it
// touches any memory that a kernel may write.
__device__ __forceinline__ void let_successor_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void await_predecessor() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void begin_after_predecessor() {
  let_successor_start();
  await_predecessor();
}

// ---- host --------------------------------------------------------------------------------------------------------
inline int train_rc(cudaError_t e) {
  if (e == cudaSuccess) return REGTOPK_OK;
  cudaGetLastError();
  return e == cudaErrorNoDevice || e == cudaErrorInsufficientDriver || e == cudaErrorNoKernelImageForDevice
             ? REGTOPK_ERR_NO_DEVICE : REGTOPK_ERR_CUDA;
}

// Launches a kernel as described at begin_after_predecessor, in clusters of kCtas blocks.
template <int kCtas = 1, typename... Params, typename... Args>
int start(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = kCtas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = kCtas > 1 ? 2 : 1;
  return train_rc(cudaLaunchKernelEx(&cfg, kernel, args...));
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
  memset(d, 0, sizeof *d);
  d->scale = 1.0f;
  if (!p) return true;
  if (!(p->p >= 0.0 && p->p <= 1.0)) return false;
  d->threshold = (u32)rint(65536.0 * p->p);
  d->scale = d->threshold < 65536u ? (float)(65536.0 / (65536.0 - d->threshold)) : 0.0f;
  d->subsequence = p->subsequence;
  for (u32 i = 0; i < 10; ++i) {
    d->keys[2 * i] = (u32)p->seed + i * 0x9E3779B9u;
    d->keys[2 * i + 1] = (u32)(p->seed >> 32) + i * 0xBB67AE85u;
  }
  return true;
}

inline size_t type_size(int32_t t) { return t == REGTOPK_TYPE_F32 ? 4 : t == REGTOPK_TYPE_BF16 || t == REGTOPK_TYPE_F16 ? 2 : 0; }

// Whether every row of the matrix begins where eight of its elements can be read or written at once (NULL: no matrix).
inline bool rows_aligned(const void* p, int64_t ld, size_t size, int64_t rows) {
  return !p || ((uintptr_t)p % (8 * size) == 0 && (rows <= 1 || ld % 8 == 0));
}

inline bool good_matrix(const void* p, int64_t ld, int64_t rows, int64_t cols, size_t size) {
  return p && (uintptr_t)p % size == 0 && (rows <= 1 || ld >= cols);
}

// Whether a kernel of this source file ever gave up on the current device: 1 or 0, or a negative code.
inline int gave_up(cudaStream_t s) {
  unsigned int v = 0;
  const int rc = train_rc(cudaMemcpyFromSymbolAsync(&v, g_gave_up, sizeof v, 0, cudaMemcpyDeviceToHost, s));
  const int sync = train_rc(cudaStreamSynchronize(s));
  return rc != REGTOPK_OK ? rc : sync != REGTOPK_OK ? sync : (int)(v != 0);
}

}  // namespace

int regtopk_norm_gave_up(cudaStream_t s);  // dropout_norm.cu's
int regtopk_rms_gave_up(cudaStream_t s);   // rms_norm.cu's
#endif
