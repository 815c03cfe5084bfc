// The tokens' way into the order of their (worker, expert) groups and back, with its gradient (include/regtopk_experts.h).
//
// Memory traffic is the floor.  Tokens are the ones that a thread goes by, and not the sorted rows: then a token's row, its place
// numbers and weights are read once, and the rows of its experts, which lie anywhere, are whole rows that are written, or read, once.
// 16,384 rows of 2,048 bfloat16 columns to four experts each: 52 us, 6.4 TB/s; back on a float32 stream: 84 us, 6.4 TB/s.

#include "rows8.cuh"

namespace {

constexpr int kMoveThreads = 256, kMoveWarps = kMoveThreads / 32;

struct MoveArgs {
  const void* in;            // spread: the tokens, or values of their 8-bit rows; join: the sorted rows; backward: dout
  const uint8_t* in_scales;
  const void* other;         // join: residual, or NULL; backward: the sorted rows
  const int32_t* place;
  const float* weights;
  const int64_t* filled;     // NULL: no row is cleared
  void* out;
  float* dweights;
  int64_t ld_in, ld_scales, ld_other, ld_out, tokens, rows, cols;
  Divisor pieces;            // of a row: threads (VEC) or warps
  u32 total;                 // of this launch
  int k, team;               // team: warps of a token (backward)
  bool clears;               // this launch clears the rows behind the last
};

__device__ __forceinline__ bool in_rows(int32_t p, int64_t rows) { return p >= 0 && p < rows; }

// Zeros to the rows from *filled on, by all threads of the grid.
template <typename T, bool VEC> __device__ __forceinline__ void clear_tail(const MoveArgs& a) {
  if (!a.filled || !a.clears) return;
  int64_t first = *a.filled;
  first = first < 0 ? 0 : first > a.rows ? a.rows : first;
  const int64_t threads = (int64_t)gridDim.x * kMoveThreads, own = (int64_t)blockIdx.x * kMoveThreads + threadIdx.x;
  const int64_t pieces = VEC ? a.cols / 8 : a.cols;
  for (int64_t i = own; i < (a.rows - first) * pieces; i += threads) {
    const int64_t r = i / pieces, c = i - r * pieces;
    T* to = static_cast<T*>(a.out) + (first + r) * a.ld_out;
    if (VEC) {
      Eight<T> v;
      v.clear();
      v.store(to + c * 8);
    } else {
      to[c] = from_float<T>(0.0f);
    }
  }
}

// Which token and which of its columns: VEC: a thread has eight neighbours; otherwise a warp has 256 columns.
template <bool VEC> struct Piece {
  int64_t token;
  int c0, lane;
  bool there;
  __device__ __forceinline__ Piece(const MoveArgs& a) {
    const u32 at = blockIdx.x * (VEC ? kMoveThreads : kMoveWarps) + (VEC ? threadIdx.x : threadIdx.x >> 5);
    const u32 r = a.pieces.quotient_of(at);
    there = at < a.total;
    token = r;
    c0 = (int)(at - r * a.pieces.d) * (VEC ? 8 : 256);
    lane = VEC ? 0 : threadIdx.x & 31;
  }
};

template <typename T, bool PACKED, bool WHOLE> __device__ __forceinline__ void spread_apart(const MoveArgs& a, int64_t token, int c0, int lane, int cols) {
  const int first = c0 + lane, left = cols - first;
  Octet f;
  if (PACKED) read_rows8_apart<WHOLE>(f, static_cast<const uint8_t*>(a.in) + token * a.ld_in + first, a.in_scales + token * a.ld_scales + (c0 >> 5), lane, left);
  else read_apart<T, WHOLE>(f, static_cast<const T*>(a.in) + token * a.ld_in + first, left);
  for (int j = 0; j < a.k; ++j) {
    const int32_t p = a.place[token * a.k + j];
    if (in_rows(p, a.rows)) store_apart<T, WHOLE>(f, static_cast<T*>(a.out) + (int64_t)p * a.ld_out + first, left);
  }
}

template <typename T, bool PACKED, bool VEC> __global__ void __launch_bounds__(kMoveThreads) k_spread(const __grid_constant__ MoveArgs a) {
  begin_after_predecessor();
  const Piece<VEC> at(a);
  const int cols = (int)a.cols;
  if (VEC && at.there) {
    Eight<T> v;
    if (PACKED) {
      Octet f;
      Packed8 p;
      p.fetch(static_cast<const uint8_t*>(a.in) + at.token * a.ld_in + at.c0, a.in_scales + at.token * a.ld_scales + (at.c0 >> 5));
      p.get(f);
      v.put(f);
    } else {
      v.fetch(static_cast<const T*>(a.in) + at.token * a.ld_in + at.c0);
    }
    const int32_t* place = a.place + at.token * a.k;
    for (int j = 0; j < a.k; ++j) {
      const int32_t p = place[j];
      if (in_rows(p, a.rows)) v.store(static_cast<T*>(a.out) + (int64_t)p * a.ld_out + at.c0);
    }
  } else if (at.there) {
    if (cols - at.c0 >= 256) spread_apart<T, PACKED, true>(a, at.token, at.c0, at.lane, cols);
    else spread_apart<T, PACKED, false>(a, at.token, at.c0, at.lane, cols);
  }
  clear_tail<T, VEC>(a);
}

template <typename T, typename O, bool VEC, bool WHOLE> __device__ __forceinline__ void join_piece(const MoveArgs& a, int64_t token, int c0, int lane, int cols) {
  // Rows under way: of unaligned 16-bit types two, whose fewer registers leave room for more warps (8,192 tokens of 2,047 bfloat16 columns
  // from four rows each 54 us, with four 65 us).
  constexpr int kJoinStep = VEC || sizeof(T) == 4 ? 4 : 2;
  const int first = c0 + lane, left = cols - first;
  const int32_t* place = a.place + token * a.k;
  const float* weights = a.weights + token * a.k;
  Octet sum;
#pragma unroll
  for (int i = 0; i < 4; ++i) sum[i] = both(0.0f);
  for (int j0 = 0; j0 < a.k; j0 += kJoinStep) {
    int32_t p[kJoinStep];
    float w[kJoinStep];
#pragma unroll
    for (int j = 0; j < kJoinStep; ++j) {
      p[j] = j0 + j < a.k ? place[j0 + j] : -1;
      w[j] = !a.weights ? 1.0f : j0 + j < a.k ? weights[j0 + j] : 0.0f;
    }
    Octet f[kJoinStep];
#pragma unroll
    for (int j = 0; j < kJoinStep; ++j) {
      const bool there = in_rows(p[j], a.rows);
      const T* row = static_cast<const T*>(a.in) + (there ? (int64_t)p[j] * a.ld_in : 0);
      if (VEC) read_eight<T, VEC, false>(f[j], row, c0, lane, there ? cols : 0);
      else if (WHOLE && there) read_apart<T, true>(f[j], row + first, left);
      else read_apart<T, false>(f[j], row + first, there ? left : 0);
      if (!there) w[j] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < kJoinStep; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] = fma2(f[j][i], both(w[j]), sum[i]);
  }
  if (a.other) {
    Octet r;
    const O* row = static_cast<const O*>(a.other) + token * a.ld_other;
    if (VEC) read_eight<O, VEC, false>(r, row, c0, lane, cols);
    else read_apart<O, WHOLE>(r, row + first, left);
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = add2(sum[i], r[i]);
  }
  O* out = static_cast<O*>(a.out) + token * a.ld_out;
  if (VEC) store_eight<O, VEC>(sum, out, c0, lane, cols);
  else store_apart<O, WHOLE>(sum, out + first, left);
}

template <typename T, typename O, bool VEC> __global__ void __launch_bounds__(kMoveThreads) k_join(const __grid_constant__ MoveArgs a) {
  begin_after_predecessor();
  const Piece<VEC> at(a);
  if (!at.there) return;
  const int cols = (int)a.cols;
  if (!VEC && cols - at.c0 >= 256) join_piece<T, O, VEC, true>(a, at.token, at.c0, at.lane, cols);
  else join_piece<T, O, VEC, false>(a, at.token, at.c0, at.lane, cols);
}

// Products of a token's dout with one of its rows, and what that row's gradient is.
template <typename T> __device__ __forceinline__ float back_of(Octet& f, const Octet& d, float w) {
  float2 s = both(0.0f);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    s = fma2(f[i], d[i], s);
    f[i] = mul2(d[i], both(w));
  }
  return s.x + s.y;
}
// 256 columns of a token's dout and of STEP of its rows, unaligned.
template <typename T, typename D, int STEP, bool WHOLE>
__device__ __forceinline__ void back_apart(const MoveArgs& a, const D* dout, const int64_t (&to)[STEP], const float (&w)[STEP], float (&dot)[STEP], int first,
                                           int left) {
  Octet d, f[STEP];
  read_apart<D, WHOLE>(d, dout + first, left);
#pragma unroll
  for (int j = 0; j < STEP; ++j)
    if (to[j] >= 0) read_apart<T, WHOLE>(f[j], static_cast<const T*>(a.other) + to[j] * a.ld_other + first, left);
#pragma unroll
  for (int j = 0; j < STEP; ++j) {
    if (to[j] < 0) continue;
    dot[j] += back_of<T>(f[j], d, w[j]);
    store_apart<T, WHOLE>(f[j], static_cast<T*>(a.out) + to[j] * a.ld_out + first, left);
  }
}
// The columns c, c + step, ... of an aligned row, eight neighbours at a time; the next ones are on their way while these are worked on.
template <typename T, typename D, int STEP>
__device__ __forceinline__ void back_aligned(const MoveArgs& a, const D* dout, const int64_t (&to)[STEP], const float (&w)[STEP], float (&dot)[STEP], int c,
                                             int step, int cols) {
  Eight<D> next_d;
  Eight<T> next_f[STEP];
  const auto fetch = [&](int at) {
    next_d.fetch(dout + at);
#pragma unroll
    for (int j = 0; j < STEP; ++j)
      if (to[j] >= 0) next_f[j].fetch(static_cast<const T*>(a.other) + to[j] * a.ld_other + at);
  };
  if (c < cols) fetch(c);
  for (; c < cols; c += step) {
    Octet d, f[STEP];
    next_d.get(d);
#pragma unroll
    for (int j = 0; j < STEP; ++j) next_f[j].get(f[j]);
    if (c + step < cols) fetch(c + step);
#pragma unroll
    for (int j = 0; j < STEP; ++j) {
      if (to[j] < 0) continue;
      dot[j] += back_of<T>(f[j], d, w[j]);
      Eight<T> v;
      v.put(f[j]);
      v.store(static_cast<T*>(a.out) + to[j] * a.ld_out + c);
    }
  }
}

// A team of warps a token: its warps share the row's units of 256 columns, and each has STEP of the token's rows under way beside
// dout.  8,192 tokens of 2,048 columns, four rows each: bfloat16 55 us with three blocks an SM (58.5 us with two), binary32 93 us with two
// (108 us with three, which spill); 2,047 bfloat16 columns 83 us with STEP 2 and four blocks (110 us with 4 and two).
template <typename T, typename D, bool VEC, int STEP> __global__ void __launch_bounds__(kMoveThreads, sizeof(T) == 4 ? 2 : VEC ? 3 : 4) k_join_back(const __grid_constant__ MoveArgs a) {
  __shared__ float part[kMoveWarps][STEP];
  begin_after_predecessor();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, member = warp % a.team, teams = kMoveWarps / a.team;
  const int64_t t = (int64_t)blockIdx.x * teams + warp / a.team;
  const bool there = t < a.tokens;
  for (int j0 = 0; j0 < a.k; j0 += STEP) {
    int64_t to[STEP];  // where each row is, -1: nowhere
    float w[STEP], dot[STEP];
#pragma unroll
    for (int j = 0; j < STEP; ++j) {
      const bool used = there && j0 + j < a.k;
      const int32_t p = used ? a.place[t * a.k + j0 + j] : -1;
      to[j] = in_rows(p, a.rows) ? p : -1;
      w[j] = used ? a.weights[t * a.k + j0 + j] : 0.0f;
      dot[j] = 0.0f;
    }
    if (there) {
      const int cols = (int)a.cols;
      const D* dout = static_cast<const D*>(a.in) + t * a.ld_in;
      if (VEC) {
        back_aligned<T, D, STEP>(a, dout, to, w, dot, member * 256 + lane * 8, a.team * 256, cols);
      } else {
        for (int c0 = member * 256; c0 < cols; c0 += a.team * 256) {
          if (cols - c0 >= 256) back_apart<T, D, STEP, true>(a, dout, to, w, dot, c0 + lane, cols - c0 - lane);
          else back_apart<T, D, STEP, false>(a, dout, to, w, dot, c0 + lane, cols - c0 - lane);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < STEP; ++j) {
      const float s = warp_sum(dot[j]);
      if (lane == 0) part[warp][j] = s;
    }
    if (a.team > 1) __syncthreads();
    else __syncwarp();
    if (member == 0 && lane < STEP && there && j0 + lane < a.k) {
      float s = 0.0f;
      for (int i = 0; i < a.team; ++i) s += part[warp + i][lane];
      a.dweights[t * a.k + j0 + lane] = s;
    }
    if (a.team > 1) __syncthreads();
    else __syncwarp();
  }
  clear_tail<T, VEC>(a);
}

// ---- launches --------------------------------------------------------------------------------------------------------
constexpr int64_t kMostCols = (int64_t)1 << 30, kMostPieces = ((int64_t)1 << 31) - kMoveThreads;

// launch(args, grid) for as many tokens at a time as have fewer than 2^31 pieces.
template <typename Launch> int in_parts(MoveArgs a, bool vec, size_t in_size, size_t other_size, size_t out_size, const Launch& launch) {
  const int64_t pieces = vec ? a.cols / 8 : (a.cols + 255) / 256, tokens = a.tokens, most = kMostPieces / pieces;
  const u32 per = vec ? kMoveThreads : kMoveWarps;
  a.pieces = divisor(pieces);
  int64_t done = 0;
  do {
    a.tokens = tokens - done < most ? tokens - done : most;
    a.total = (u32)(a.tokens * pieces);
    a.clears = done == 0;
    const unsigned blocks = (a.total + per - 1) / per;
    const int rc = launch(a, blocks ? blocks : 1u);
    if (rc != REGTOPK_OK) return rc;
    done += a.tokens;
    a.in = static_cast<const char*>(a.in) + a.tokens * a.ld_in * (int64_t)in_size;
    if (a.in_scales) a.in_scales += a.tokens * a.ld_scales;
    if (a.other) a.other = static_cast<const char*>(a.other) + a.tokens * a.ld_other * (int64_t)other_size;
    a.place += a.tokens * a.k;
    if (a.weights) a.weights += a.tokens * a.k;
    a.out = static_cast<char*>(a.out) + a.tokens * a.ld_out * (int64_t)out_size;
  } while (done < tokens);
  return REGTOPK_OK;
}

template <typename T, typename D, int STEP> int launch_join_back_step(const MoveArgs& a, bool vec, unsigned grid, cudaStream_t s) {
  if (vec) return start(k_join_back<T, D, true, STEP>, grid, kMoveThreads, 0, s, a);
  return start(k_join_back<T, D, false, (sizeof(T) == 2 && STEP > 2 ? 2 : STEP)>, grid, kMoveThreads, 0, s, a);
}
template <typename T, typename D> int launch_join_back(const MoveArgs& a, bool vec, unsigned grid, cudaStream_t s) {
  return a.k == 1 ? launch_join_back_step<T, D, 1>(a, vec, grid, s) : a.k == 2 ? launch_join_back_step<T, D, 2>(a, vec, grid, s)
                                                                               : launch_join_back_step<T, D, 4>(a, vec, grid, s);
}

inline bool bad_shape(int64_t tokens, int32_t k, int64_t rows, int64_t cols) {
  return tokens < 0 || k < 1 || rows < 0 || cols < 0 || cols > kMostCols || tokens > INT64_MAX / 64;
}

}  // namespace

#define REGTOPK_BY_TYPE(call) \
  (type == REGTOPK_TYPE_F32 ? call(float) : type == REGTOPK_TYPE_BF16 ? call(__nv_bfloat16) : call(__half))
#define REGTOPK_BY_TYPES(call, second)                                                                            \
  (type == REGTOPK_TYPE_F32    ? call(float, float)                                                               \
   : type == REGTOPK_TYPE_BF16 ? (second == type ? call(__nv_bfloat16, __nv_bfloat16) : call(__nv_bfloat16, float)) \
   : second == type            ? call(__half, __half)                                                             \
                               : call(__half, float))

extern "C" {

int regtopk_spread_tokens(const void* x, int64_t ldx, const uint8_t* scales, int64_t ld_scales, const int32_t* place,
                          const int64_t* filled, void* out, int64_t ld_out, int64_t tokens, int32_t k, int64_t rows, int64_t cols,
                          int32_t type, void* cuda_stream) {
  const size_t size = type_size(type);
  if (!size || bad_shape(tokens, k, rows, cols) || (uintptr_t)filled % 8) return REGTOPK_ERR_INVALID_ARG;
  if (k > REGTOPK_ROUTE_MAX_CHOICES) return REGTOPK_ERR_TOO_LARGE;
  if (rows == 0 || cols == 0) return REGTOPK_OK;
  if (!good_matrix(out, ld_out, rows, cols, size)) return REGTOPK_ERR_INVALID_ARG;
  if (tokens > 0 && (!good_matrix(place, k, 1, k, 4) || (scales ? !good_rows8(static_cast<const uint8_t*>(x), ldx, scales, ld_scales, tokens, cols, 1)
                                                                : !good_matrix(x, ldx, tokens, cols, size)))) return REGTOPK_ERR_INVALID_ARG;
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  MoveArgs a = {};
  a.in = x; a.ld_in = ldx; a.in_scales = scales; a.ld_scales = ld_scales; a.place = place; a.filled = filled; a.out = out; a.ld_out = ld_out;
  a.tokens = tokens; a.rows = rows; a.cols = cols; a.k = k;
  const bool vec = cols % 8 == 0 && rows_aligned(out, ld_out, size, rows) &&
                   (scales ? rows8_aligned(static_cast<const uint8_t*>(x), ldx, tokens) : rows_aligned(x, ldx, size, tokens));
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return in_parts(a, vec, scales ? 1 : size, 0, 0, [&](const MoveArgs& part, unsigned grid) {
#define REGTOPK_SPREAD(T)                                                                                         \
  (scales ? (vec ? start(k_spread<T, true, true>, grid, kMoveThreads, 0, s, part) : start(k_spread<T, true, false>, grid, kMoveThreads, 0, s, part)) \
          : (vec ? start(k_spread<T, false, true>, grid, kMoveThreads, 0, s, part) : start(k_spread<T, false, false>, grid, kMoveThreads, 0, s, part)))
    return REGTOPK_BY_TYPE(REGTOPK_SPREAD);
#undef REGTOPK_SPREAD
  });
}

int regtopk_join_tokens(const void* from, int64_t ld_from, const int32_t* place, const float* weights, const void* residual,
                        int64_t ld_residual, void* out, int64_t ld_out, int64_t tokens, int32_t k, int64_t rows, int64_t cols,
                        int32_t type, int32_t out_type, void* cuda_stream) {
  const size_t size = type_size(type), osize = type_size(out_type);
  if (!size || !osize || (out_type != type && out_type != REGTOPK_TYPE_F32) || bad_shape(tokens, k, rows, cols) || (uintptr_t)weights % 4)
    return REGTOPK_ERR_INVALID_ARG;
  if (k > REGTOPK_ROUTE_MAX_CHOICES) return REGTOPK_ERR_TOO_LARGE;
  if (tokens == 0 || cols == 0) return REGTOPK_OK;
  if (!good_matrix(out, ld_out, tokens, cols, osize) || !good_matrix(place, k, 1, k, 4) || (rows > 0 && !good_matrix(from, ld_from, rows, cols, size)) ||
      (residual && !good_matrix(residual, ld_residual, tokens, cols, osize))) return REGTOPK_ERR_INVALID_ARG;
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  MoveArgs a = {};
  a.in = from; a.ld_in = ld_from; a.other = residual; a.ld_other = ld_residual; a.place = place; a.weights = weights; a.out = out; a.ld_out = ld_out;
  a.tokens = tokens; a.rows = rows; a.cols = cols; a.k = k;
  const bool vec = cols % 8 == 0 && rows_aligned(from, ld_from, size, rows) && rows_aligned(out, ld_out, osize, tokens) &&
                   rows_aligned(residual, ld_residual, osize, tokens);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return in_parts(a, vec, 0, osize, osize, [&](const MoveArgs& part, unsigned grid) {
#define REGTOPK_JOIN(T, O) (vec ? start(k_join<T, O, true>, grid, kMoveThreads, 0, s, part) : start(k_join<T, O, false>, grid, kMoveThreads, 0, s, part))
    return REGTOPK_BY_TYPES(REGTOPK_JOIN, out_type);
#undef REGTOPK_JOIN
  });
}

int regtopk_join_tokens_backward(const void* dout, int64_t ld_dout, const void* from, int64_t ld_from, const int32_t* place,
                                 const float* weights, const int64_t* filled, void* dfrom, int64_t ld_dfrom, float* dweights,
                                 int64_t tokens, int32_t k, int64_t rows, int64_t cols, int32_t type, int32_t dout_type,
                                 void* cuda_stream) {
  const size_t size = type_size(type), dsize = type_size(dout_type);
  if (!size || !dsize || (dout_type != type && dout_type != REGTOPK_TYPE_F32) || bad_shape(tokens, k, rows, cols) || (uintptr_t)filled % 8)
    return REGTOPK_ERR_INVALID_ARG;
  if (k > REGTOPK_ROUTE_MAX_CHOICES || tokens > INT32_MAX) return REGTOPK_ERR_TOO_LARGE;
  if (rows > 0 && cols > 0 && (!good_matrix(from, ld_from, rows, cols, size) || !good_matrix(dfrom, ld_dfrom, rows, cols, size))) return REGTOPK_ERR_INVALID_ARG;
  if (tokens > 0 && (!good_matrix(place, k, 1, k, 4) || !good_matrix(weights, k, 1, k, 4) || !good_matrix(dweights, k, 1, k, 4) ||
                     (cols > 0 && !good_matrix(dout, ld_dout, tokens, cols, dsize)))) return REGTOPK_ERR_INVALID_ARG;
  if (tokens == 0 && (rows == 0 || cols == 0)) return REGTOPK_OK;
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  MoveArgs a = {};
  a.in = dout; a.ld_in = ld_dout; a.other = from; a.ld_other = ld_from; a.place = place; a.weights = weights; a.filled = filled;
  a.out = dfrom; a.ld_out = ld_dfrom; a.dweights = dweights; a.tokens = tokens; a.rows = cols ? rows : 0; a.cols = cols; a.k = k; a.clears = true;
  const bool vec = cols % 8 == 0 && rows_aligned(dout, ld_dout, dsize, tokens) && rows_aligned(from, ld_from, size, rows) && rows_aligned(dfrom, ld_dfrom, size, rows);
  // As many warps a token as it has units, while that makes no more than four times the warps that the device holds at once (300 bfloat16 tokens of
  // 4,096 columns, four rows each, 8.9 us, with one warp a token 13.8 us; 2,000 of 1,023 10.7 us and 14.7 us; 5,003 float16 ones of 777 columns, two rows
  // each, 11.3 us either way; all with the rows in L2).
  const int64_t units = (cols + 255) / 256;
  a.team = 1;
  while (a.team < kMoveWarps && a.team < units && tokens * a.team * 2 <= (int64_t)sms * 32 * 4) a.team *= 2;
  const int64_t teams = kMoveWarps / a.team, blocks = tokens ? (tokens + teams - 1) / teams : 1;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
#define REGTOPK_JOIN_BACK(T, D) launch_join_back<T, D>(a, vec, (unsigned)blocks, s)
  return REGTOPK_BY_TYPES(REGTOPK_JOIN_BACK, dout_type);
#undef REGTOPK_JOIN_BACK
}

}  // extern "C"
