// Gated activations with their gradients, their input kept in 8 bits, and 8-bit rows alone (include/regtopk_experts.h).
//
// Memory traffic is their floor: each reads its inputs once and writes its outputs once, and nothing is kept for the backward
// pass but the 8-bit rows (1 + 1/32 bytes for an element, where the activation's input has two): it forms the activation
// and its slope again from them, and the output, which the next product's weight gradients need, on the way.
// 32,768 rows of 2,304 bfloat16 columns, gated silu: 98 us forward with the 8-bit rows, 6.2 TB/s, 122 us back, 6.2 TB/s.  Binary32, 8,192 x 2,048,
// ungated, both ways: silu 60 us, gelu 67 us (86 us with CUDA's erfc).

#include "rows8.cuh"

namespace {

constexpr int kActThreads = 256;

// ---- f(x) = x p(x) and its slope ---------------------------------------------------------------------------------
// FAST, for 16-bit types: exponentials and reciprocals are the hardware's approximations, and the argument of an exponential is rounded, which
// 2^-16 of p covers down to 2^-40, 2^-15 further down; the types' own rounding is 2^-9 and 2^-12.

// p = 1 / (1 + exp(-x)) and q = 1 - p, without cancellation; an infinite exponential gives 0 and 1.
template <bool FAST> __device__ __forceinline__ void logistic(float x, float& p, float& q) {
  const float e = FAST ? exp2_fast(-kLog2E * x) : expf(-x);
  p = FAST ? reciprocal_fast(1.0f + e) : 1.0f / (1.0f + e);
  q = FAST || x < 0.0f ? 1.0f - p : e * p;  // what 1 - p loses for large x is 2^-23 x, x at most 17, where p is not 1
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
    float e;  // exp(-x^2 / 2)
    if (FAST) {
      e = exp2_fast(-0.5f * kLog2E * x * x);
      // Phi(-|x|) = e t S(t), t = 1 / (1 + 0.31 |x|); S is a fit like the one below, 2^-17.7 relative for |x| up to 14.6: relative, because f(x) keeps as
      // many bits for large negative x as for others (a formula with one term less whose absolute error is small was 0.4 % off at -5.5 and 1 % at -8).
      const float t = reciprocal_fast(fmaf(0.31f, fabsf(x), 1.0f));
      float h = fmaf(-0.0739291694f, t, 0.180450416f);
      h = fmaf(h, t, 0.0157446378f);
      h = fmaf(h, t, 0.133429822f);
      h = fmaf(h, t, 0.120441268f);
      h = fmaf(h, t, 0.123860704f);
      h = h * t * e;
      p = x >= 0.0f ? 1.0f - h : h;
    } else {
      // Near 0 Phi is 1/2 + x R(x^2), so that its error is that of the sum; further out Phi(-|x|) = e t S(t), t = 1 / (1 + 0.28 |x|), whose error is relative
      // to it.  R and S are fits of least largest error, made by linear programming over Chebyshev nodes against the scaled erfc in binary64: 2^-30 and
      // 2^-29 of Phi(-|x|), for |x| up to 1 and from 1 to 14.6.  e gets back what x^2 has lost by rounding.  In all at most
      // 12 units of 2^-24 of Phi (2^-20 is what tests hold it to), and in the mean less than one.
      const float w = fminf(fmaxf(x, -16.0f), 16.0f), square = w * w;  // past 15 Phi is 0 or 1 in binary32, and x^2 may overflow
      e = expf(-0.5f * square);
      e = fmaf(-0.5f * fmaf(w, w, -square), e, e);
      float r = fmaf(-7.4629199e-06f, square, 0.000112952245f);
      r = fmaf(r, square, -0.00118578506f);
      r = fmaf(r, square, 0.00997307842f);
      r = fmaf(r, square, -0.0664903144f);
      r = fmaf(r, square, 0.398942278f);
      const float middle = fmaf(x, r, 0.5f);
      const float t = reciprocal_fast(fmaf(0.28f, fabsf(w), 1.0f));
      float h = fmaf(0.0316852507f, t, -0.121061593f);
      h = fmaf(h, t, 0.137709857f);
      h = fmaf(h, t, -0.0469639849f);
      h = fmaf(h, t, 0.0941641724f);
      h = fmaf(h, t, 0.0768444794f);
      h = fmaf(h, t, 0.104344522f);
      h = fmaf(h, t, 0.111574424f);
      h = fmaf(h, t, 0.111709031f);
      h = h * t * e;
      p = fabsf(x) < 1.0f ? middle : x >= 0.0f ? 1.0f - h : h;
    }
    if (slope) *slope = fmaf(x, 0.3989422804f * e, p);
  }
  return x * p;
}

// ---- where a thread's columns lie ------------------------------------------------------------------------------------
// VEC: rows are aligned and have a multiple of eight columns; a thread has kActStep times eight neighbours, four threads share a block
// of 32, and the threads go through all rows' blocks one after the other.  Otherwise a warp has 256 columns of a row, every 32nd a
// lane's.
struct Layout {
  int64_t cols, row0;  // row0: where this launch begins
  Divisor pieces;      // of a row: groups of eight columns (VEC), or of 256
  u32 total;           // of this launch, fewer than 2^31
};
constexpr int kActStep = 2;  // with one the gradient of 32,768 x 2,304 waits for memory: 142 us, with two 122 us

template <bool VEC> struct Spot {
  int64_t row;
  int c0;
  bool there;
  __device__ __forceinline__ Spot(const Layout& l, u32 at) {
    const u32 r = l.pieces.quotient_of(at);
    c0 = (int)(at - r * l.pieces.d) * (VEC ? 8 : 256);
    there = at < l.total && c0 < (int)l.cols;
    row = l.row0 + (at < l.total ? r : 0);
  }
};
template <bool VEC> __device__ __forceinline__ u32 first_piece() {
  return VEC ? blockIdx.x * (kActThreads * kActStep) + threadIdx.x : blockIdx.x * (kActThreads / 32) + (threadIdx.x >> 5);
}

// ---- kernels -------------------------------------------------------------------------------------------------------
struct ActArgs {
  Layout at;
  const void *a, *dy;
  const uint8_t* in_scales;    // of a, where it is 8-bit rows
  void *y, *da;                // y NULL: not written
  uint8_t *values, *scales;    // forward: NULL: not kept
  int64_t lda, ldy, ld_dy, ld_da, ld_in_scales, ld_values, ld_scales, half_blocks;
};

template <typename T, int KIND, bool GATED> __device__ __forceinline__ void forward_of(Octet& x, const Octet& u) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = make_float2(activate<KIND, sizeof(T) == 2>(x[i].x, nullptr), activate<KIND, sizeof(T) == 2>(x[i].y, nullptr));
    if (GATED) x[i] = mul2(x[i], u[i]);
  }
}

template <typename T, int KIND, bool GATED, bool WHOLE>
__device__ __forceinline__ void forward_apart(const ActArgs& a, int64_t row, int c0, int cols) {
  const int lane = threadIdx.x & 31, first = c0 + lane, left = cols - first;
  const T* from = static_cast<const T*>(a.a) + row * a.lda + first;
  Octet x, u;
  read_apart<T, WHOLE>(x, from, left);
  if (GATED) read_apart<T, WHOLE>(u, from + cols, left);
  if (a.values) {
    uint8_t *values = a.values + row * a.ld_values + first, *scales = a.scales + row * a.ld_scales + (c0 >> 5);
    store_rows8_apart<WHOLE>(x, values, scales, lane, left);
    if (GATED) store_rows8_apart<WHOLE>(u, values + cols, scales + a.half_blocks, lane, left);
  }
  forward_of<T, KIND, GATED>(x, u);
  store_apart<T, WHOLE>(x, static_cast<T*>(a.y) + row * a.ldy + first, left);
}

template <typename T, int KIND, bool GATED, bool VEC>
__global__ void __launch_bounds__(kActThreads) k_activation(const __grid_constant__ ActArgs a) {
  begin_after_predecessor();
  const int cols = (int)a.at.cols;
  if constexpr (VEC) {
    Eight<T> x[kActStep], u[kActStep];
#pragma unroll
    for (int n = 0; n < kActStep; ++n) {
      const Spot<true> at(a.at, first_piece<true>() + n * kActThreads);
      const T* from = static_cast<const T*>(a.a) + at.row * a.lda + at.c0;
      x[n].clear();
      u[n].clear();
      if (at.there) x[n].fetch(from);
      if (GATED && at.there) u[n].fetch(from + cols);
    }
#pragma unroll
    for (int n = 0; n < kActStep; ++n) {
      const Spot<true> at(a.at, first_piece<true>() + n * kActThreads);
      Octet f, g;
      x[n].get(f);
      u[n].get(g);
      if (a.values) {
        uint8_t *values = a.values + at.row * a.ld_values + at.c0, *scales = a.scales + at.row * a.ld_scales + (at.c0 >> 5);
        store_rows8(f, values, scales, at.there);
        if (GATED) store_rows8(g, values + cols, scales + a.half_blocks, at.there);
      }
      forward_of<T, KIND, GATED>(f, g);
      x[n].put(f);
      if (at.there) x[n].store(static_cast<T*>(a.y) + at.row * a.ldy + at.c0);
    }
  } else {
    const Spot<false> at(a.at, first_piece<false>());
    if (!at.there) return;
    if (cols - at.c0 >= 256) forward_apart<T, KIND, GATED, true>(a, at.row, at.c0, cols);
    else forward_apart<T, KIND, GATED, false>(a, at.row, at.c0, cols);
  }
}

// x and u become the gradients to the halves, d the output.
template <typename T, int KIND, bool GATED> __device__ __forceinline__ void backward_of(Octet& x, Octet& u, Octet& d) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float2 slope, f = make_float2(activate<KIND, sizeof(T) == 2>(x[i].x, &slope.x), activate<KIND, sizeof(T) == 2>(x[i].y, &slope.y));
    x[i] = mul2(slope, d[i]);
    if (GATED) {
      const float2 up = u[i];
      x[i] = mul2(x[i], up);
      u[i] = mul2(d[i], f);
      d[i] = mul2(up, f);
    } else {
      d[i] = f;
    }
  }
}

template <typename T, int KIND, bool GATED, bool KEPT8, bool WHOLE>
__device__ __forceinline__ void backward_apart(const ActArgs& a, int64_t row, int c0, int cols) {
  const int lane = threadIdx.x & 31, first = c0 + lane, left = cols - first;
  Octet d, x, u;
  if (KEPT8) {
    const uint8_t *from = static_cast<const uint8_t*>(a.a) + row * a.lda + first, *scales = a.in_scales + row * a.ld_in_scales + (c0 >> 5);
    read_rows8_apart<WHOLE>(x, from, scales, lane, left);
    if (GATED) read_rows8_apart<WHOLE>(u, from + cols, scales + a.half_blocks, lane, left);
  } else {
    const T* from = static_cast<const T*>(a.a) + row * a.lda + first;
    read_apart<T, WHOLE>(x, from, left);
    if (GATED) read_apart<T, WHOLE>(u, from + cols, left);
  }
  read_apart<T, WHOLE>(d, static_cast<const T*>(a.dy) + row * a.ld_dy + first, left);
  backward_of<T, KIND, GATED>(x, u, d);
  T* da = static_cast<T*>(a.da) + row * a.ld_da + first;
  store_apart<T, WHOLE>(x, da, left);
  if (GATED) store_apart<T, WHOLE>(u, da + cols, left);
  if (a.y) store_apart<T, WHOLE>(d, static_cast<T*>(a.y) + row * a.ldy + first, left);
}

template <typename T, int KIND, bool GATED, bool KEPT8, bool VEC>
__global__ void __launch_bounds__(kActThreads) k_activation_back(const __grid_constant__ ActArgs a) {
  begin_after_predecessor();
  const int cols = (int)a.at.cols;
  if constexpr (VEC) {
    Octet d, x, u;
    Eight<T> in[kActStep], wide_x[KEPT8 ? 1 : kActStep], wide_u[KEPT8 ? 1 : kActStep];
    Packed8 packed_x[KEPT8 ? kActStep : 1], packed_u[KEPT8 ? kActStep : 1];
#pragma unroll
    for (int n = 0; n < kActStep; ++n) {
      const Spot<true> at(a.at, first_piece<true>() + n * kActThreads);
      if (KEPT8) {
        const uint8_t *from = static_cast<const uint8_t*>(a.a) + at.row * a.lda + at.c0, *scales = a.in_scales + at.row * a.ld_in_scales + (at.c0 >> 5);
        packed_x[n].clear();
        packed_u[n].clear();
        if (at.there) packed_x[n].fetch(from, scales);
        if (GATED && at.there) packed_u[n].fetch(from + cols, scales + a.half_blocks);
      } else {
        const T* from = static_cast<const T*>(a.a) + at.row * a.lda + at.c0;
        wide_x[n].clear();
        wide_u[n].clear();
        if (at.there) wide_x[n].fetch(from);
        if (GATED && at.there) wide_u[n].fetch(from + cols);
      }
      in[n].clear();
      if (at.there) in[n].fetch(static_cast<const T*>(a.dy) + at.row * a.ld_dy + at.c0);
    }
#pragma unroll
    for (int n = 0; n < kActStep; ++n) {
      const Spot<true> at(a.at, first_piece<true>() + n * kActThreads);
      in[n].get(d);
      if (KEPT8) {
        packed_x[n].get(x);
        if (GATED) packed_u[n].get(u);
      } else {
        wide_x[n].get(x);
        if (GATED) wide_u[n].get(u);
      }
      backward_of<T, KIND, GATED>(x, u, d);
      if (!at.there) continue;
      T* da = static_cast<T*>(a.da) + at.row * a.ld_da + at.c0;
      in[n].put(x);
      in[n].store(da);
      if (GATED) {
        in[n].put(u);
        in[n].store(da + cols);
      }
      if (a.y) {
        in[n].put(d);
        in[n].store(static_cast<T*>(a.y) + at.row * a.ldy + at.c0);
      }
    }
  } else {
    const Spot<false> at(a.at, first_piece<false>());
    if (!at.there) return;
    if (cols - at.c0 >= 256) backward_apart<T, KIND, GATED, KEPT8, true>(a, at.row, at.c0, cols);
    else backward_apart<T, KIND, GATED, KEPT8, false>(a, at.row, at.c0, cols);
  }
}

template <typename T, bool VEC> __global__ void __launch_bounds__(kActThreads) k_pack8(const __grid_constant__ ActArgs a) {
  begin_after_predecessor();
  Octet f;
  if constexpr (VEC) {
    Eight<T> x[kActStep];
#pragma unroll
    for (int n = 0; n < kActStep; ++n) {
      const Spot<true> at(a.at, first_piece<true>() + n * kActThreads);
      x[n].clear();
      if (at.there) x[n].fetch(static_cast<const T*>(a.a) + at.row * a.lda + at.c0);
    }
#pragma unroll
    for (int n = 0; n < kActStep; ++n) {
      const Spot<true> at(a.at, first_piece<true>() + n * kActThreads);
      x[n].get(f);
      store_rows8(f, a.values + at.row * a.ld_values + at.c0, a.scales + at.row * a.ld_scales + (at.c0 >> 5), at.there);
    }
  } else {
    const Spot<false> at(a.at, first_piece<false>());
    if (!at.there) return;
    const int lane = threadIdx.x & 31, first = at.c0 + lane, left = (int)a.at.cols - first;
    read_apart<T, false>(f, static_cast<const T*>(a.a) + at.row * a.lda + first, left);
    store_rows8_apart<false>(f, a.values + at.row * a.ld_values + first, a.scales + at.row * a.ld_scales + (at.c0 >> 5), lane, left);
  }
}

template <typename T, bool VEC> __global__ void __launch_bounds__(kActThreads) k_unpack8(const __grid_constant__ ActArgs a) {
  begin_after_predecessor();
  Octet f;
  if constexpr (VEC) {
    Packed8 v[kActStep];
#pragma unroll
    for (int n = 0; n < kActStep; ++n) {
      const Spot<true> at(a.at, first_piece<true>() + n * kActThreads);
      v[n].clear();
      if (at.there) v[n].fetch(static_cast<const uint8_t*>(a.a) + at.row * a.lda + at.c0, a.in_scales + at.row * a.ld_in_scales + (at.c0 >> 5));
    }
#pragma unroll
    for (int n = 0; n < kActStep; ++n) {
      const Spot<true> at(a.at, first_piece<true>() + n * kActThreads);
      v[n].get(f);
      Eight<T> x;
      x.put(f);
      if (at.there) x.store(static_cast<T*>(a.y) + at.row * a.ldy + at.c0);
    }
  } else {
    const Spot<false> at(a.at, first_piece<false>());
    if (!at.there) return;
    const int lane = threadIdx.x & 31, first = at.c0 + lane, left = (int)a.at.cols - first;
    read_rows8_apart<false>(f, static_cast<const uint8_t*>(a.a) + at.row * a.lda + first, a.in_scales + at.row * a.ld_in_scales + (at.c0 >> 5), lane, left);
    store_apart<T, false>(f, static_cast<T*>(a.y) + at.row * a.ldy + first, left);
  }
}

// ---- launches --------------------------------------------------------------------------------------------------------
// `launch` for as many rows at a time as have fewer than 2^31 pieces.
template <typename Launch> int in_parts(ActArgs a, bool vec, int64_t rows, int64_t cols, const Launch& launch) {
  const int64_t pieces = vec ? 4 * blocks_of(cols) : (cols + 255) / 256, most = (((int64_t)1 << 31) - kActThreads * kActStep) / pieces;
  const u32 per = vec ? kActThreads * kActStep : kActThreads / 32;
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
