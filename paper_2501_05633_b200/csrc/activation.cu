// Gated activations with their gradients, their input kept in 8 bits, and 8-bit rows alone (include/regtopk_experts.h).
//
// Memory traffic is their floor: each reads its inputs once and writes its outputs once, and nothing is kept for the backward
// pass but the 8-bit rows (1 + 1/32 bytes for an element, where the activation's input has two): it forms the activation
// and its slope again from them, and the output, which the next product's weight gradients need, on the way.

#include "rows8.cuh"

namespace {

constexpr int kActThreads = 256;

// ---- f(x) = x p(x) and its slope ---------------------------------------------------------------------------------
// exp and 1 / (1 + t), t in [0, 1].  FAST, for 16-bit types: the hardware's approximations, off by 2^-20 where they matter.
template <bool FAST> __device__ __forceinline__ float exp_of(float x) { return FAST ? __expf(x) : expf(x); }
template <bool FAST> __device__ __forceinline__ float over(float t) { return FAST ? __fdividef(1.0f, t) : 1.0f / t; }

// p = 1 / (1 + exp(-x)) and q = 1 - p, both from exp(-|x|), so that neither overflows nor cancels.
template <bool FAST> __device__ __forceinline__ void logistic(float x, float& p, float& q) {
  const float t = exp_of<FAST>(-fabsf(x)), r = over<FAST>(1.0f + t), s = t * r;
  p = x >= 0.0f ? r : s;
  q = x >= 0.0f ? s : r;
}

// f(x) = x p; slope: f'(x) too.
template <int KIND, bool FAST> __device__ __forceinline__ float activate(float x, float* slope) {
  float p, q;
  if (KIND == REGTOPK_ACTIVATION_SILU) {
    logistic<FAST>(x, p, q);
    if (slope) *slope = p * fmaf(x, q, 1.0f);
  } else if (KIND == REGTOPK_ACTIVATION_GELU_TANH) {
    // (1 + tanh z) / 2 = 1 / (1 + exp(-2z)).  Past 16 p is 0 or 1 in binary32, and x^3 may overflow.
    const float c = 1.5957691216057308f, w = fminf(fmaxf(x, -16.0f), 16.0f), w2 = w * w;
    logistic<FAST>(c * fmaf(0.044715f * w2, w, w), p, q);
    if (slope) *slope = fmaf(x * (p * q), c * fmaf(0.134145f, w2, 1.0f), p);
  } else {
    const float e = exp_of<FAST>(-0.5f * x * x);
    if (FAST) {
      // Phi(-|x|) by approximation 7.1.26 of Abramowitz and Stegun (Hastings), off by 7.5e-8: six terms and one exponential that
      // the slope needs anyway.
      const float t = over<true>(fmaf(0.23164189f, fabsf(x), 1.0f));
      float h = fmaf(1.061405429f, t, -1.453152027f);
      h = fmaf(h, t, 1.421413741f);
      h = fmaf(h, t, -0.284496736f);
      h = fmaf(h, t, 0.254829592f);
      h = 0.5f * h * t * e;
      p = x >= 0.0f ? 1.0f - h : h;
    } else {
      // erfc(z + r), r what z = -x / sqrt(2) has lost by rounding: without it p is off by z^2 units of 2^-22
      const float z = -0.70710677f * x, r = fmaf(-1.2101617e-8f, x, fmaf(-0.70710677f, x, -z));
      p = fmaf(-0.56418958f * e, r, 0.5f * erfcf(z));
    }
    if (slope) *slope = fmaf(x, 0.3989422804f * e, p);
  }
  return x * p;
}

// ---- where a thread's eight columns lie ----------------------------------------------------------------------------
// VEC: rows are aligned and have a multiple of eight columns; a thread has eight neighbours, four threads a block of 32, and
// the threads go through all rows' blocks one after the other.  Otherwise a warp has 256 columns of a row, and each lane every 32nd.
struct Layout {
  int64_t cols, row0;  // row0: where this launch begins
  Divisor pieces;      // of a row: threads (VEC) or warps
  u32 total;           // of this launch, fewer than 2^31
};
template <bool VEC> struct Spot {
  int64_t row, c0;
  int lane;
  bool there;
  __device__ __forceinline__ Spot(const Layout& l) {
    const u32 at = blockIdx.x * (VEC ? kActThreads : kActThreads / 32) + (VEC ? threadIdx.x : threadIdx.x >> 5);
    const u32 r = l.pieces.quotient_of(at);
    there = at < l.total;
    row = l.row0 + (there ? r : 0);
    c0 = (int64_t)(at - r * l.pieces.d) * (VEC ? 8 : 256);
    lane = VEC ? 0 : threadIdx.x & 31;
  }
};
// ---- kernels -------------------------------------------------------------------------------------------------------
struct ActArgs {
  Layout at;
  const void *a, *dy;
  const uint8_t* in_scales;    // of a, where it is 8-bit rows
  void *y, *da;                // y NULL: not written
  uint8_t *values, *scales;    // forward: NULL: not kept
  int64_t lda, ldy, ld_dy, ld_da, ld_in_scales, ld_values, ld_scales, half_blocks;
};

template <typename T, int KIND, bool GATED, bool VEC>
__global__ void __launch_bounds__(kActThreads) k_activation(const __grid_constant__ ActArgs a) {
  begin_after_predecessor();
  const Spot<VEC> at(a.at);
  const int64_t cols = at.there ? a.at.cols : 0;
  const T* row = static_cast<const T*>(a.a) + at.row * a.lda;
  Octet x, u;
  read_eight<T, VEC, false>(x, row, at.c0, at.lane, cols);
  if (GATED) read_eight<T, VEC, false>(u, row + a.at.cols, at.c0, at.lane, cols);
  if (a.values) {
    uint8_t *values = a.values + at.row * a.ld_values, *scales = a.scales + at.row * a.ld_scales;
    store_rows8<VEC>(x, values, scales, at.c0, at.lane, cols);
    if (GATED) store_rows8<VEC>(u, values + a.at.cols, scales + a.half_blocks, at.c0, at.lane, cols);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = make_float2(activate<KIND, sizeof(T) == 2>(x[i].x, nullptr), activate<KIND, sizeof(T) == 2>(x[i].y, nullptr));
    if (GATED) x[i] = mul2(x[i], u[i]);
  }
  store_eight<T, VEC>(x, static_cast<T*>(a.y) + at.row * a.ldy, at.c0, at.lane, cols);
}

template <typename T, int KIND, bool GATED, bool KEPT8, bool VEC>
__global__ void __launch_bounds__(kActThreads) k_activation_back(const __grid_constant__ ActArgs a) {
  begin_after_predecessor();
  const Spot<VEC> at(a.at);
  const int64_t cols = at.there ? a.at.cols : 0;
  Octet d, x, u;
  if (KEPT8) {
    const uint8_t *row = static_cast<const uint8_t*>(a.a) + at.row * a.lda, *scales = a.in_scales + at.row * a.ld_in_scales;
    read_rows8<VEC>(x, row, scales, at.c0, at.lane, cols);
    if (GATED) read_rows8<VEC>(u, row + a.at.cols, scales + a.half_blocks, at.c0, at.lane, cols);
  } else {
    const T* row = static_cast<const T*>(a.a) + at.row * a.lda;
    read_eight<T, VEC, false>(x, row, at.c0, at.lane, cols);
    if (GATED) read_eight<T, VEC, false>(u, row + a.at.cols, at.c0, at.lane, cols);
  }
  read_eight<T, VEC, false>(d, static_cast<const T*>(a.dy) + at.row * a.ld_dy, at.c0, at.lane, cols);
  Octet slope;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    x[i] = make_float2(activate<KIND, sizeof(T) == 2>(x[i].x, &slope[i].x), activate<KIND, sizeof(T) == 2>(x[i].y, &slope[i].y));
  T* da = static_cast<T*>(a.da) + at.row * a.ld_da;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    slope[i] = mul2(slope[i], d[i]);
    if (GATED) {
      slope[i] = mul2(slope[i], u[i]);
      u[i] = mul2(u[i], x[i]);  // the output
      d[i] = mul2(d[i], x[i]);  // the gradient to the second half
    }
  }
  store_eight<T, VEC>(slope, da, at.c0, at.lane, cols);
  if (GATED) store_eight<T, VEC>(d, da + a.at.cols, at.c0, at.lane, cols);
  if (a.y) store_eight<T, VEC>(GATED ? u : x, static_cast<T*>(a.y) + at.row * a.ldy, at.c0, at.lane, cols);
}

template <typename T, bool VEC> __global__ void __launch_bounds__(kActThreads) k_pack8(const __grid_constant__ ActArgs a) {
  begin_after_predecessor();
  const Spot<VEC> at(a.at);
  const int64_t cols = at.there ? a.at.cols : 0;
  Octet x;
  read_eight<T, VEC, false>(x, static_cast<const T*>(a.a) + at.row * a.lda, at.c0, at.lane, cols);
  store_rows8<VEC>(x, a.values + at.row * a.ld_values, a.scales + at.row * a.ld_scales, at.c0, at.lane, cols);
}

template <typename T, bool VEC> __global__ void __launch_bounds__(kActThreads) k_unpack8(const __grid_constant__ ActArgs a) {
  begin_after_predecessor();
  const Spot<VEC> at(a.at);
  const int64_t cols = at.there ? a.at.cols : 0;
  Octet x;
  read_rows8<VEC>(x, static_cast<const uint8_t*>(a.a) + at.row * a.lda, a.in_scales + at.row * a.ld_in_scales, at.c0, at.lane, cols);
  store_eight<T, VEC>(x, static_cast<T*>(a.y) + at.row * a.ldy, at.c0, at.lane, cols);
}

// ---- launches --------------------------------------------------------------------------------------------------------
// `launch` for as many rows at a time as have fewer than 2^31 pieces.
template <typename Launch> int in_parts(ActArgs a, bool vec, int64_t rows, int64_t cols, const Launch& launch) {
  const int64_t pieces = vec ? 4 * blocks_of(cols) : (cols + 255) / 256, most = (((int64_t)1 << 31) - kActThreads) / pieces;
  const u32 per = vec ? kActThreads : kActThreads / 32;
  a.at.cols = cols;
  a.at.pieces = divisor(pieces);
  for (a.at.row0 = 0; a.at.row0 < rows; a.at.row0 += most) {
    a.at.total = (u32)((rows - a.at.row0 < most ? rows - a.at.row0 : most) * pieces);
    const int rc = launch(a, (a.at.total + per - 1) / per);
    if (rc != REGTOPK_OK) return rc;
  }
  return REGTOPK_OK;
}
template <typename T, int KIND, bool GATED> int launch_act(const ActArgs& a, bool vec, unsigned grid, cudaStream_t s) {
  return vec ? start(k_activation<T, KIND, GATED, true>, grid, kActThreads, 0, s, a) : start(k_activation<T, KIND, GATED, false>, grid, kActThreads, 0, s, a);
}
template <typename T, int KIND, bool GATED> int launch_act_back(const ActArgs& a, bool vec, unsigned grid, cudaStream_t s) {
  if (a.in_scales)
    return vec ? start(k_activation_back<T, KIND, GATED, true, true>, grid, kActThreads, 0, s, a)
               : start(k_activation_back<T, KIND, GATED, true, false>, grid, kActThreads, 0, s, a);
  return vec ? start(k_activation_back<T, KIND, GATED, false, true>, grid, kActThreads, 0, s, a)
             : start(k_activation_back<T, KIND, GATED, false, false>, grid, kActThreads, 0, s, a);
}
template <typename T> int launch_pack8(const ActArgs& a, bool vec, unsigned grid, cudaStream_t s) {
  return vec ? start(k_pack8<T, true>, grid, kActThreads, 0, s, a) : start(k_pack8<T, false>, grid, kActThreads, 0, s, a);
}
template <typename T> int launch_unpack8(const ActArgs& a, bool vec, unsigned grid, cudaStream_t s) {
  return vec ? start(k_unpack8<T, true>, grid, kActThreads, 0, s, a) : start(k_unpack8<T, false>, grid, kActThreads, 0, s, a);
}

constexpr int64_t kMostCols = (int64_t)1 << 30;

}  // namespace

#define REGTOPK_BY_TYPE(call) \
  (type == REGTOPK_TYPE_F32 ? call(float) : type == REGTOPK_TYPE_BF16 ? call(__nv_bfloat16) : call(__half))
#define REGTOPK_BY_KIND(call, T)                                                                                          \
  (kind == REGTOPK_ACTIVATION_SILU   ? (gated ? call(T, REGTOPK_ACTIVATION_SILU, true) : call(T, REGTOPK_ACTIVATION_SILU, false)) \
   : kind == REGTOPK_ACTIVATION_GELU ? (gated ? call(T, REGTOPK_ACTIVATION_GELU, true) : call(T, REGTOPK_ACTIVATION_GELU, false)) \
                                     : (gated ? call(T, REGTOPK_ACTIVATION_GELU_TANH, true) : call(T, REGTOPK_ACTIVATION_GELU_TANH, false)))

extern "C" {

int regtopk_pack8(const void* x, int64_t ldx, uint8_t* values, int64_t ld_values, uint8_t* scales, int64_t ld_scales,
                  int64_t rows, int64_t cols, int32_t type, void* cuda_stream) {
  const size_t size = type_size(type);
  if (!size || rows < 0 || cols < 0 || cols > kMostCols) return REGTOPK_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return REGTOPK_OK;
  if (!good_matrix(x, ldx, rows, cols, size) || !good_rows8(values, ld_values, scales, ld_scales, rows, cols, 1)) return REGTOPK_ERR_INVALID_ARG;
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  ActArgs a = {};
  const bool vec = cols % 8 == 0 && rows_aligned(x, ldx, size, rows) && rows8_aligned(values, ld_values, rows);
  a.a = x; a.lda = ldx; a.values = values; a.ld_values = ld_values; a.scales = scales; a.ld_scales = ld_scales;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
#define REGTOPK_PACK(T) launch_pack8<T>(part, vec, grid, s)
  return in_parts(a, vec, rows, cols, [&](const ActArgs& part, unsigned grid) { return REGTOPK_BY_TYPE(REGTOPK_PACK); });
#undef REGTOPK_PACK
}

int regtopk_unpack8(const uint8_t* values, int64_t ld_values, const uint8_t* scales, int64_t ld_scales, void* x, int64_t ldx,
                    int64_t rows, int64_t cols, int32_t type, void* cuda_stream) {
  const size_t size = type_size(type);
  if (!size || rows < 0 || cols < 0 || cols > kMostCols) return REGTOPK_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return REGTOPK_OK;
  if (!good_matrix(x, ldx, rows, cols, size) || !good_rows8(values, ld_values, scales, ld_scales, rows, cols, 1)) return REGTOPK_ERR_INVALID_ARG;
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  ActArgs a = {};
  const bool vec = cols % 8 == 0 && rows_aligned(x, ldx, size, rows) && rows8_aligned(values, ld_values, rows);
  a.a = values; a.lda = ld_values; a.in_scales = scales; a.ld_in_scales = ld_scales; a.y = x; a.ldy = ldx;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
#define REGTOPK_UNPACK(T) launch_unpack8<T>(part, vec, grid, s)
  return in_parts(a, vec, rows, cols, [&](const ActArgs& part, unsigned grid) { return REGTOPK_BY_TYPE(REGTOPK_UNPACK); });
#undef REGTOPK_UNPACK
}

int regtopk_activation(const void* x, int64_t lda, void* y, int64_t ldy, uint8_t* values, int64_t ld_values, uint8_t* scales,
                       int64_t ld_scales, int64_t rows, int64_t cols, int32_t kind, int32_t gated, int32_t type, void* cuda_stream) {
  const size_t size = type_size(type);
  const int halves = gated ? 2 : 1;
  if (!size || rows < 0 || cols < 0 || cols > kMostCols || kind < 0 || kind > REGTOPK_ACTIVATION_GELU_TANH) return REGTOPK_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return REGTOPK_OK;
  if (!good_matrix(x, lda, rows, halves * cols, size) || !good_matrix(y, ldy, rows, cols, size) || (!values != !scales) ||
      (values && !good_rows8(values, ld_values, scales, ld_scales, rows, cols, halves))) return REGTOPK_ERR_INVALID_ARG;
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  ActArgs a = {};
  const bool vec = cols % 8 == 0 && rows_aligned(x, lda, size, rows) && rows_aligned(y, ldy, size, rows) && rows8_aligned(values, ld_values, rows);
  a.a = x; a.lda = lda; a.y = y; a.ldy = ldy; a.values = values; a.ld_values = ld_values; a.scales = scales; a.ld_scales = ld_scales;
  a.half_blocks = blocks_of(cols);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
#define REGTOPK_ACT(T, K, G) launch_act<T, K, G>(part, vec, grid, s)
#define REGTOPK_ACT_OF(T) REGTOPK_BY_KIND(REGTOPK_ACT, T)
  return in_parts(a, vec, rows, cols, [&](const ActArgs& part, unsigned grid) { return REGTOPK_BY_TYPE(REGTOPK_ACT_OF); });
#undef REGTOPK_ACT_OF
#undef REGTOPK_ACT
}

int regtopk_activation_backward(const void* dy, int64_t ld_dy, const void* x, int64_t lda, const uint8_t* in_scales, int64_t ld_scales,
                                void* da, int64_t ld_da, void* y, int64_t ldy, int64_t rows, int64_t cols, int32_t kind, int32_t gated,
                                int32_t type, void* cuda_stream) {
  const size_t size = type_size(type);
  const int halves = gated ? 2 : 1;
  if (!size || rows < 0 || cols < 0 || cols > kMostCols || kind < 0 || kind > REGTOPK_ACTIVATION_GELU_TANH) return REGTOPK_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return REGTOPK_OK;
  const uint8_t* values = in_scales ? static_cast<const uint8_t*>(x) : nullptr;
  if (!good_matrix(dy, ld_dy, rows, cols, size) || !good_matrix(da, ld_da, rows, halves * cols, size) ||
      !(in_scales ? good_rows8(values, lda, in_scales, ld_scales, rows, cols, halves) : good_matrix(x, lda, rows, halves * cols, size)) ||
      (y && !good_matrix(y, ldy, rows, cols, size))) return REGTOPK_ERR_INVALID_ARG;
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  ActArgs a = {};
  const bool vec = cols % 8 == 0 && rows_aligned(dy, ld_dy, size, rows) && rows_aligned(da, ld_da, size, rows) && rows_aligned(y, ldy, size, rows) &&
                   (in_scales ? rows8_aligned(values, lda, rows) : rows_aligned(x, lda, size, rows));
  a.a = x; a.lda = lda; a.in_scales = in_scales; a.ld_in_scales = ld_scales; a.dy = dy; a.ld_dy = ld_dy; a.da = da; a.ld_da = ld_da;
  a.y = y; a.ldy = ldy; a.half_blocks = blocks_of(cols);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
#define REGTOPK_ACT_BACK(T, K, G) launch_act_back<T, K, G>(part, vec, grid, s)
#define REGTOPK_ACT_BACK_OF(T) REGTOPK_BY_KIND(REGTOPK_ACT_BACK, T)
  return in_parts(a, vec, rows, cols, [&](const ActArgs& part, unsigned grid) { return REGTOPK_BY_TYPE(REGTOPK_ACT_BACK_OF); });
#undef REGTOPK_ACT_BACK_OF
#undef REGTOPK_ACT_BACK
}

}  // extern "C"
