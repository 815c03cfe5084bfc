// Root-mean-square norm, behind a residual sum and with an output in 8 bits, and its gradient (include/regtopk_experts.h).
//
// As for the layer norm, one read and one write of each array is the floor, and the same rings bring a team's rows through shared
// memory.  There is one sum to a row in either direction, so a row costs one exchange between its warps.  32,768 rows of 1,024 bfloat16
// columns on a binary32 stream: 70 us, 5.7 TB/s, with 8-bit rows beside y 78 us; the gradient of 8,192 rows of 4,096 bfloat16 columns with a
// second gradient: 55 us and 4 for the sum over blocks, 4.6 TB/s, bound by latency at the sixteen warps whose rows an SM's shared memory holds.

#include "rows8.cuh"

namespace {

// ---- forward ---------------------------------------------------------------------------------------------------------
struct RmsArgs {
  Source source[3];  // x, residual
  const float* weight;
  void *y, *h;
  uint8_t *values, *scales;
  float* rstd;
  int64_t ldy, ldh, ld_values, ld_scales, rows;
  int cols, wide;
  float eps;
  RingShape ring;
};

template <typename T, typename S, bool VEC, int U, bool RING>
__global__ void __maxnreg__(U <= 2 ? 80 : 128) k_rms(const __grid_constant__ RmsArgs a) {
  extern __shared__ __align__(16) char smem[];
  __shared__ Common common;
  const Team t(a.ring.warps, U);
  begin_after_predecessor();
  float* weight = reinterpret_cast<float*>(smem);
  const int64_t first = (int64_t)blockIdx.x * a.ring.teams + t.index, step = (int64_t)gridDim.x * a.ring.teams;
  Ring<true> ring = make_ring<RING, true>(common, a.ring, a.source, reinterpret_cast<char*>(weight + padded(a.cols)), t, first, step, a.rows);
  if (RING) {
    fetch_vector<VEC>(weight, a.weight, a.cols);
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
  }
  const float per_col = 1.0f / (float)a.cols;
  u32 turn = 0;
  for (int64_t row = first; row < a.rows; row += step, turn ^= 1) {
    if (RING) ring.await(t.leads());
    Octet f[U];
    float2 square = both(0.0f);
    const T* x = ring.row_of<T, VEC, RING>(row, 0);
    const S* residual = ring.row_of<S, VEC, RING>(row, 1);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c0 = t.col0 + u * 256;
      read_eight<T, VEC, RING>(f[u], x, c0, t.lane, a.cols);
      if (a.ring.row_bytes[1]) {
        Octet r;
        read_eight<S, VEC, RING>(r, residual, c0, t.lane, a.cols);
#pragma unroll
        for (int i = 0; i < 4; ++i) f[u][i] = add2(f[u][i], r[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) square = fma2(f[u][i], f[u][i], square);  // zeros past the end
    }
    float sum = warp_sum(square.x + square.y);
    if (t.warps > 1 && t.lane == 0) common.exchange[turn][t.index * t.warps + t.warp].x = sum;
    if (RING || t.warps > 1) t.sync();  // the row has been read by all
    if (RING) ring.pass(row, t.leads());
    if (t.warps > 1) {
      const float2* v = &common.exchange[turn][t.index * t.warps];
      sum = 0.0f;
      for (int i = 0; i < t.warps; ++i) sum += v[i].x;
    }
    const float rstd = inverse_root(fmaf(sum, per_col, a.eps));
    if (t.leads()) a.rstd[row] = rstd;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c0 = t.col0 + u * 256;
      if (c0 >= a.cols) break;
      if (a.h) store_eight<S, VEC>(f[u], static_cast<S*>(a.h) + row * a.ldh, c0, t.lane, a.cols);
      Octet w;
      if (RING) read_vector<VEC>(w, weight, c0, t.lane);
      else load_vector<VEC>(w, a.weight, a.wide, c0, t.lane, a.cols);
#pragma unroll
      for (int i = 0; i < 4; ++i) f[u][i] = mul2(mul2(f[u][i], both(rstd)), w[i]);
      if (a.y) store_eight<T, VEC>(f[u], static_cast<T*>(a.y) + row * a.ldy, c0, t.lane, a.cols);
      if (a.values) {
        uint8_t *values = a.values + row * a.ld_values, *scales = a.scales + row * a.ld_scales;
        if (VEC) store_rows8(f[u], values + c0 + t.lane * 8, scales + ((c0 + t.lane * 8) >> 5), c0 + t.lane * 8 < a.cols);
        else store_rows8_apart<false>(f[u], values + c0 + t.lane, scales + (c0 >> 5), t.lane, a.cols - c0 - t.lane);
      }
    }
  }
}

// ---- backward --------------------------------------------------------------------------------------------------------
struct RmsBackArgs {
  Source source[3];  // dy, h, dh
  const float *rstd, *weight;
  void *dx, *dres;
  int64_t ld_dx, ld_dres, rows, block_rows;
  int cols, groups, wide;
  const int64_t* offsets;  // NULL: one group of all rows
  float* partial;          // [blocks + groups][cols], or NULL: no weight gradient
  RingShape ring;
};

// A block takes `block_rows` rows in a row and leaves the sums for each group that it meets in the slot (block + group) of the
// partial sums, which no other block has (with ascending groups block + group only grows).
template <typename T, typename S, bool VEC, int U, bool RING>
__global__ void __launch_bounds__(32 * kMostWarps, 1) k_rms_back(const __grid_constant__ RmsBackArgs a) {
  extern __shared__ __align__(16) char smem[];
  __shared__ Common common;
  const Team t(a.ring.warps, U);
  begin_after_predecessor();
  float *weight = reinterpret_cast<float*>(smem), *joint = weight + padded(a.cols);  // joint: the teams' sums, if there are two or more
  const int64_t r0 = blockIdx.x * a.block_rows, r1 = min(a.rows, r0 + a.block_rows), first = r0 + t.index, step = a.ring.teams;
  Ring<false> ring = make_ring<RING, false>(common, a.ring, a.source, reinterpret_cast<char*>(joint + (a.ring.teams > 1 ? padded(a.cols) : 0)), t, first, step, r1);
  if (RING) fetch_vector<VEC>(weight, a.weight, a.cols);
  int g = a.partial ? group_of(a.offsets, a.groups, r0, a.rows, t.lane) : a.groups;
  float rstd = first < r1 ? a.rstd[first] : 0.0f;
  if (RING) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
  }
  const float inv = 1.0f / (float)a.cols;
  u32 turn = 0;
  int64_t row = first;
  for (int64_t at = r0; at < r1;) {
    // rows [at, end) belong to one group, or to none
    int64_t end = r1;
    bool counted = false;
    if (g < a.groups) {
      const int64_t lo = offset_at(a.offsets, g, a.rows), hi = offset_at(a.offsets, g + 1, a.rows);
      if (at < lo) {
        end = min(lo, r1);
      } else if (at < hi) {
        end = min(hi, r1);
        counted = true;
      } else {
        ++g;
        continue;
      }
    }
    Octet dw[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) dw[u][i] = both(0.0f);
    for (; row < end; row += step, turn ^= 1) {
      const float next_rstd = row + step < r1 ? a.rstd[row + step] : 0.0f;
      if (RING) ring.await(t.leads());
      const T* dy = ring.row_of<T, VEC, RING>(row, 0);
      const S* h = ring.row_of<S, VEC, RING>(row, 1);
      float2 sum = both(0.0f);
      // What has been read stays in registers where they suffice, three or four units of 16-bit types as they lie in memory: then the row's
      // place is free after one barrier (8,192 rows of 4,096 bfloat16 columns 65 -> 59 us).
      constexpr bool kRaw = VEC && RING && U > 2 && sizeof(T) + sizeof(S) == 4, kKeeps = !RING || kRaw || U <= 2;
      constexpr int kKept = kKeeps ? U : 1;
      Octet kept_g[kRaw ? 1 : kKept], kept_u[kRaw ? 1 : kKept], kept_r[kRaw || !RING ? 1 : kKept];
      Eight<T> raw_d[kRaw ? U : 1];
      Eight<S> raw_h[kRaw ? U : 1], raw_r[kRaw ? U : 1];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c0 = t.col0 + u * 256;
        if (c0 >= a.cols) break;
        Octet &g8 = kept_g[kRaw ? 0 : u % kKept], &v = kept_u[kRaw ? 0 : u % kKept], w;
        if constexpr (kRaw) {  // zeros past the end
          const int c = c0 + t.lane * 8;
          raw_d[u].clear();
          raw_h[u].clear();
          raw_r[u].clear();
          if (c < a.cols) {
            raw_d[u].load(dy + c);
            raw_h[u].load(h + c);
            if (a.ring.row_bytes[2]) raw_r[u].load(ring.row_of<S, VEC, RING>(row, 2) + c);
          }
          raw_d[u].get(g8);
          raw_h[u].get(v);
        } else {
          read_eight<T, VEC, RING>(g8, dy, c0, t.lane, a.cols);
          read_eight<S, VEC, RING>(v, h, c0, t.lane, a.cols);
          if (RING && kKeeps && a.ring.row_bytes[2]) read_eight<S, VEC, RING>(kept_r[u % kKept], ring.row_of<S, VEC, RING>(row, 2), c0, t.lane, a.cols);
        }
        if (RING) read_vector<VEC>(w, weight, c0, t.lane);
        else load_vector<VEC>(w, a.weight, a.wide, c0, t.lane, a.cols);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = mul2(v[i], both(rstd));
          dw[u][i] = fma2(g8[i], v[i], dw[u][i]);
          g8[i] = mul2(g8[i], w[i]);
          sum = fma2(g8[i], v[i], sum);
        }
      }
      float m = warp_sum(sum.x + sum.y);
      if (t.warps > 1 && t.lane == 0) common.exchange[turn][t.index * t.warps + t.warp].x = m;
      if (t.warps > 1 || (RING && kKeeps)) t.sync();  // the row has been read by all, if it is kept
      if (RING && kKeeps) ring.pass(row, t.leads());
      if (t.warps > 1) {
        const float2* v = &common.exchange[turn][t.index * t.warps];
        m = 0.0f;
        for (int i = 0; i < t.warps; ++i) m += v[i].x;
      }
      m *= -inv;
      if (RING) asm volatile("" ::: "memory");  // what follows is read, or converted, again: kept, it would not fit the registers
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c0 = t.col0 + u * 256;
        if (c0 >= a.cols) break;
        Octet &d = kept_g[kRaw ? 0 : u % kKept], &v = kept_u[kRaw ? 0 : u % kKept];
        if (kRaw || !kKeeps) {
          Octet w;
          if constexpr (kRaw) {
            raw_d[u].get(d);
            raw_h[u].get(v);
          } else {
            read_eight<T, VEC, RING>(d, dy, c0, t.lane, a.cols);
            read_eight<S, VEC, RING>(v, h, c0, t.lane, a.cols);
          }
          read_vector<VEC>(w, weight, c0, t.lane);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            d[i] = mul2(d[i], w[i]);
            v[i] = mul2(v[i], both(rstd));
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = mul2(fma2(v[i], both(m), d[i]), both(rstd));
        if (a.ring.row_bytes[2]) {
          Octet& r = kept_r[kRaw || !RING ? 0 : u % kKept];
          if constexpr (kRaw) raw_r[u].get(r);
          else if (!RING || !kKeeps) read_eight<S, VEC, RING>(r, ring.row_of<S, VEC, RING>(row, 2), c0, t.lane, a.cols);
#pragma unroll
          for (int i = 0; i < 4; ++i) d[i] = add2(d[i], r[i]);
        }
        if (a.dres) store_eight<S, VEC>(d, static_cast<S*>(a.dres) + row * a.ld_dres, c0, t.lane, a.cols);
        store_eight<T, VEC>(d, static_cast<T*>(a.dx) + row * a.ld_dx, c0, t.lane, a.cols);
      }
      if (!kKeeps) {
        t.sync();
        ring.pass(row, t.leads());
      }
      rstd = next_rstd;
    }
    if (counted) {
      float* out = a.partial + (int64_t)(blockIdx.x + g) * a.cols;
      if (a.ring.teams > 1) {  // the teams add theirs one after the other, so that the order is fixed
        for (int i = 0; i < a.ring.teams; ++i) {
          if (t.index == i) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
              const int c0 = t.col0 + u * 256;
              if (c0 >= a.cols) break;
              // any place will do that a lane finds again: pair k of the lane's eight lies at k * 64 + lane * 2
              float2* w = reinterpret_cast<float2*>(joint + c0) + t.lane;
#pragma unroll
              for (int k = 0; k < 4; ++k) w[k * 32] = i ? add2(w[k * 32], dw[u][k]) : dw[u][k];
            }
          }
          __syncthreads();
        }
        for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
          const int e = c & 255, lane = VEC ? e >> 3 : e & 31, j = VEC ? e & 7 : e >> 5;
          out[c] = joint[(c & ~255) + (j >> 1) * 64 + lane * 2 + (j & 1)];
        }
        __syncthreads();
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int c = t.col0 + u * 256 + lane_col<VEC>(t.lane, j);
            if (c < a.cols) out[c] = (j & 1) ? dw[u][j >> 1].y : dw[u][j >> 1].x;
          }
      }
      ++g;
    }
    at = end;
  }
}

// The weight gradient: for each group the sum of its blocks' partial sums, kRuns runs of them side by side, always the same
// runs in the same order.
struct RmsSumArgs {
  const float* partial;
  float* dweight;
  int64_t ld_dweight, rows, block_rows;
  int cols, accumulate;
  const int64_t* offsets;
};

constexpr int kRuns = 16;
__global__ void __launch_bounds__(32 * kRuns) k_rms_sum(const RmsSumArgs a) {
  __shared__ float part[kRuns][33];
  begin_after_predecessor();
  const int g = blockIdx.y, c = blockIdx.x * 32 + threadIdx.x;
  const int64_t lo = offset_at(a.offsets, g, a.rows), hi = offset_at(a.offsets, g + 1, a.rows);
  float w = 0.0f;
  if (c < a.cols && lo < hi) {
    const int64_t last = (hi - 1) / a.block_rows;
#pragma unroll 4
    for (int64_t block = lo / a.block_rows + threadIdx.y; block <= last; block += kRuns) w += a.partial[(block + g) * a.cols + c];
  }
  part[threadIdx.y][threadIdx.x] = w;
  __syncthreads();
#pragma unroll
  for (int i = threadIdx.y; i < 32; i += kRuns) {  // each warp adds the runs of some columns, a lane a run
    const int at = blockIdx.x * 32 + i;
    const float s = warp_sum((int)threadIdx.x < kRuns ? part[threadIdx.x][i] : 0.0f);
    if (threadIdx.x == 0 && at < a.cols) {
      float* out = a.dweight + g * a.ld_dweight + at;
      *out = a.accumulate ? *out + s : s;
    }
  }
}

// ---- launches --------------------------------------------------------------------------------------------------------
template <typename T, typename S, bool VEC, int U>
int launch_rms(const RmsArgs& a, const Plan& p, int dev, int sms, cudaStream_t s) {
  const int64_t tasks = (a.rows + a.ring.teams - 1) / a.ring.teams, most = (int64_t)sms * p.blocks;
  const int blocks = (int)(tasks < most ? tasks : most);
  if (p.rings) {
    constexpr auto k = k_rms<T, S, VEC, U, true>;
    if (!allow_smem<k>(dev)) return train_rc(cudaGetLastError());
    return start(k, blocks, p.threads, p.smem, s, a);
  }
  return start(k_rms<T, S, VEC, U, false>, blocks, p.threads, 0, s, a);
}

template <typename T, typename S, bool VEC, int U>
int launch_rms_back(const RmsBackArgs& a, const Plan& p, int dev, cudaStream_t s) {
  const int blocks = (int)((a.rows + a.block_rows - 1) / a.block_rows);
  if (p.rings) {
    constexpr auto k = k_rms_back<T, S, VEC, U, true>;
    if (!allow_smem<k>(dev)) return train_rc(cudaGetLastError());
    return start(k, blocks, p.threads, p.smem, s, a);
  }
  constexpr auto k = k_rms_back<T, S, VEC, U, false>;
  if (!allow_smem<k>(dev)) return train_rc(cudaGetLastError());
  return start(k, blocks, p.threads, p.smem, s, a);
}

}  // namespace

int regtopk_rms_gave_up(cudaStream_t s) { return gave_up(s); }

// `call` with the types, the layout and the units of a warp: one of the five pairs of element and stream type.
#define REGTOPK_BY_UNITS(call, T, S, V) \
  (p.units == 1 ? call(T, S, V, 1) : p.units == 2 ? call(T, S, V, 2) : p.units == 3 ? call(T, S, V, 3) : call(T, S, V, 4))
#define REGTOPK_BY_LAYOUT(call, T, S) (vec ? REGTOPK_BY_UNITS(call, T, S, true) : REGTOPK_BY_UNITS(call, T, S, false))
#define REGTOPK_BY_TYPE(call)                                                              \
  (type == REGTOPK_TYPE_F32    ? REGTOPK_BY_LAYOUT(call, float, float)                     \
   : type == REGTOPK_TYPE_BF16 ? (stream_type == type ? REGTOPK_BY_LAYOUT(call, __nv_bfloat16, __nv_bfloat16) \
                                                      : REGTOPK_BY_LAYOUT(call, __nv_bfloat16, float))        \
   : stream_type == type       ? REGTOPK_BY_LAYOUT(call, __half, __half)                   \
                               : REGTOPK_BY_LAYOUT(call, __half, float))

extern "C" {

int regtopk_rms_norm(const void* x, int64_t ldx, const void* residual, int64_t ld_residual, const float* weight, float eps, void* y,
                     int64_t ldy, uint8_t* values, int64_t ld_values, uint8_t* scales, int64_t ld_scales, void* h, int64_t ldh,
                     float* rstd, int64_t rows, int64_t cols, int32_t type, int32_t stream_type, void* cuda_stream) {
  RmsArgs a;
  const size_t size = type_size(type), ssize = type_size(stream_type);
  if (!size || !ssize || (stream_type != type && stream_type != REGTOPK_TYPE_F32) || rows < 0 || cols < 1 || !(eps >= 0.0f && eps <= 3.4e38f))
    return REGTOPK_ERR_INVALID_ARG;
  if (cols > REGTOPK_NORM_MAX_COLS) return REGTOPK_ERR_TOO_LARGE;
  if (rows == 0) return REGTOPK_OK;
  if (!good_matrix(x, ldx, rows, cols, size) || (!y && !values) || (y && !good_matrix(y, ldy, rows, cols, size)) || (!values != !scales) ||
      (values && !good_rows8(values, ld_values, scales, ld_scales, rows, cols, 1)) ||
      (residual && !good_matrix(residual, ld_residual, rows, cols, ssize)) || (h && !good_matrix(h, ldh, rows, cols, ssize)) ||
      !good_matrix(weight, cols, 1, cols, 4) || !good_matrix(rstd, 1, 1, 1, 4)) return REGTOPK_ERR_INVALID_ARG;
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  a.source[0] = {static_cast<const char*>(x), ldx * (int64_t)size};
  a.source[1] = {static_cast<const char*>(residual), ld_residual * (int64_t)ssize};
  a.source[2] = {nullptr, 0};
  a.weight = weight; a.y = y; a.h = h; a.values = values; a.scales = scales; a.rstd = rstd; a.ldy = ldy; a.ldh = ldh;
  a.ld_values = ld_values; a.ld_scales = ld_scales; a.rows = rows; a.cols = (int)cols; a.eps = eps; a.wide = (uintptr_t)weight % 16 == 0;
  const bool vec = cols % 8 == 0 && rows_aligned(x, ldx, size, rows) && rows_aligned(y, ldy, size, rows) &&
                   rows_aligned(residual, ld_residual, ssize, rows) && rows_aligned(h, ldh, ssize, rows) && rows8_aligned(values, ld_values, rows);
  // units and blocks as for the layer norm, whose rows are read in the same way
  const Plan p = plan_of(cols, rows, {size, residual ? ssize : 0, 0}, cols <= 1024 || size + ssize == 8 ? 2 : 4, cols <= 1024 ? 3 : 2, 1, 0, sms);
  a.ring = p.ring;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
#define REGTOPK_RMS(T, S, V, U) launch_rms<T, S, V, U>(a, p, dev, sms, s)
  return REGTOPK_BY_TYPE(REGTOPK_RMS);
#undef REGTOPK_RMS
}

// A slot for each block and group.
size_t regtopk_rms_norm_backward_workspace_bytes(int64_t rows, int64_t cols, int32_t groups) {
  if (rows < 0 || cols < 1 || cols > REGTOPK_NORM_MAX_COLS || groups < 1) return 0;
  return ((rows < kMostBackBlocks ? rows : kMostBackBlocks) + (size_t)groups) * cols * sizeof(float);
}

int regtopk_rms_norm_backward(const void* dy, int64_t ld_dy, const void* h, int64_t ldh, const float* rstd, const float* weight,
                              const void* dh, int64_t ld_dh, void* dx, int64_t ld_dx, void* dresidual, int64_t ld_dresidual,
                              float* dweight, int64_t ld_dweight, const int64_t* offsets, int32_t groups, int32_t accumulate,
                              int64_t rows, int64_t cols, int32_t type, int32_t stream_type, void* workspace, size_t workspace_bytes,
                              void* cuda_stream) {
  RmsBackArgs a;
  const size_t size = type_size(type), ssize = type_size(stream_type);
  if (!size || !ssize || (stream_type != type && stream_type != REGTOPK_TYPE_F32) || rows < 0 || cols < 1 || groups < 1 ||
      (!offsets && groups != 1) || (uintptr_t)offsets % 8) return REGTOPK_ERR_INVALID_ARG;
  if (cols > REGTOPK_NORM_MAX_COLS || groups > REGTOPK_NORM_MAX_GROUPS) return REGTOPK_ERR_TOO_LARGE;
  if (dweight && !good_matrix(dweight, ld_dweight, groups, cols, 4)) return REGTOPK_ERR_INVALID_ARG;
  if (rows > 0 && (!good_matrix(dy, ld_dy, rows, cols, size) || !good_matrix(h, ldh, rows, cols, ssize) ||
                   !good_matrix(dx, ld_dx, rows, cols, size) || (dh && !good_matrix(dh, ld_dh, rows, cols, ssize)) ||
                   (dresidual && !good_matrix(dresidual, ld_dresidual, rows, cols, ssize)) ||
                   !good_matrix(weight, cols, 1, cols, 4) || !good_matrix(rstd, 1, 1, 1, 4)))
    return REGTOPK_ERR_INVALID_ARG;
  if (dweight && rows > 0) {
    if (!workspace || (uintptr_t)workspace % 16) return REGTOPK_ERR_INVALID_ARG;
    if (workspace_bytes < regtopk_rms_norm_backward_workspace_bytes(rows, cols, groups)) return REGTOPK_ERR_WORKSPACE_TOO_SMALL;
  }
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  if (sms > kMostSms) sms = kMostSms;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  a.block_rows = 1;
  if (rows > 0) {
    a.source[0] = {static_cast<const char*>(dy), ld_dy * (int64_t)size};
    a.source[1] = {static_cast<const char*>(h), ldh * (int64_t)ssize};
    a.source[2] = {static_cast<const char*>(dh), ld_dh * (int64_t)ssize};
    a.rstd = rstd; a.weight = weight; a.dx = dx; a.dres = dresidual; a.ld_dx = ld_dx; a.ld_dres = ld_dresidual;
    a.rows = rows; a.cols = (int)cols; a.wide = (uintptr_t)weight % 16 == 0; a.groups = groups; a.offsets = offsets;
    a.partial = dweight ? static_cast<float*>(workspace) : nullptr;
    // Two units a warp: with four, 8,192 rows of 4,096 bfloat16 columns take 78 us against 59 us.  Three where a row has three and is of 16-bit
    // types, so that it needs no second warp: 32,768 rows of 768 columns 39 us against 49 us.
    const Plan p = plan_of(cols, rows, {size, ssize, dh ? ssize : 0}, size + ssize == 4 && cols > 512 && cols <= 768 ? 3 : 2, 2, 1, 1, sms);
    a.ring = p.ring;
    const int64_t blocks = (int64_t)sms * (p.blocks < 4 ? p.blocks : 4), turns = (rows + blocks * p.ring.teams - 1) / (blocks * p.ring.teams);
    a.block_rows = turns * p.ring.teams;
    const bool vec = cols % 8 == 0 && rows_aligned(dy, ld_dy, size, rows) && rows_aligned(h, ldh, ssize, rows) &&
                     rows_aligned(dh, ld_dh, ssize, rows) && rows_aligned(dx, ld_dx, size, rows) &&
                     rows_aligned(dresidual, ld_dresidual, ssize, rows);
#define REGTOPK_RMS_BACK(T, S, V, U) launch_rms_back<T, S, V, U>(a, p, dev, s)
    const int rc = REGTOPK_BY_TYPE(REGTOPK_RMS_BACK);
#undef REGTOPK_RMS_BACK
    if (rc != REGTOPK_OK) return rc;
  }
  if (dweight) {
    RmsSumArgs n;
    n.partial = static_cast<const float*>(workspace); n.dweight = dweight; n.ld_dweight = ld_dweight;
    n.rows = rows; n.block_rows = a.block_rows; n.cols = (int)cols; n.accumulate = accumulate; n.offsets = offsets;
    return start(k_rms_sum, dim3((unsigned)((cols + 31) / 32), (unsigned)groups), dim3(32, kRuns), 0, s, n);
  }
  return REGTOPK_OK;
}

}  // extern "C"
