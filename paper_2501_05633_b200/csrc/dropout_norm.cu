// Dropout and layer norm with their gradients (include/regtopk_train.h).
//
// All of them are bound by memory traffic: a few operations per element and one read and one write of each array.
// So each kernel reads every input once, keeps a row in registers between its two sums and the output, and draws the
// dropout mask again wherever it is needed instead of storing it (one Philox call for eight columns costs less issue
// time than a byte of mask costs bandwidth).

#include "train_common.cuh"

namespace {

// ---- dropout -------------------------------------------------------------------------------------------------------
struct DropoutArgs {
  const void* x;
  void* y;
  int64_t ldx, ldy, rows, cols;
  Drop drop;
};

// Aligned rows of a multiple of eight columns: a thread takes groups of eight columns, kStep of them at a time so that
// that many loads are under way.
constexpr int kDropThreads = 256;
constexpr int kDropStep = 2;

template <typename T>
__global__ void __launch_bounds__(kDropThreads) k_dropout_vec(const DropoutArgs a) {
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.y);
  const int64_t groups = a.cols >> 3, total = a.rows * groups, step = (int64_t)gridDim.x * kDropThreads;
  int64_t at = (int64_t)blockIdx.x * kDropThreads + threadIdx.x;
  const int64_t row_step = step / groups, group_step = step % groups;  // so that the loop itself divides nothing
  int64_t row = at / groups, group = at % groups;
  while (at < total) {
    Eight<T> v[kDropStep];
    int64_t r[kDropStep], g[kDropStep];
#pragma unroll
    for (int i = 0; i < kDropStep; ++i) {
      r[i] = row;
      g[i] = group;
      if (at + i * step < total) v[i].load(x + row * a.ldx + group * 8);
      row += row_step;
      group += group_step;
      if (group >= groups) { group -= groups; ++row; }
    }
#pragma unroll
    for (int i = 0; i < kDropStep; ++i) {
      if (at + i * step >= total) break;
      const u32 keep = a.drop.threshold ? keep_bits(a.drop, (uint64_t)r[i], (u32)g[i]) : 0xFFu;
      Eight<T> o;
#pragma unroll
      for (int j = 0; j < 8; ++j) o.set(j, (keep >> j) & 1u ? v[i].get(j) * a.drop.scale : 0.0f);
      o.store(y + r[i] * a.ldy + g[i] * 8);
    }
    at += kDropStep * step;
  }
}

// Any other layout: a warp takes 256 columns of a row.
template <typename T>
__global__ void __launch_bounds__(kDropThreads) k_dropout_any(const DropoutArgs a) {
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.y);
  const int lane = threadIdx.x & 31;
  const int64_t units = (a.cols + 255) >> 8, total = a.rows * units;
  const int64_t step = (int64_t)gridDim.x * (kDropThreads / 32);
  for (int64_t at = (int64_t)blockIdx.x * (kDropThreads / 32) + (threadIdx.x >> 5); at < total; at += step) {
    const int64_t row = at / units, col0 = (at - row * units) << 8;
    T v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t c = col0 + lane_col<false>(lane, j);
      if (c < a.cols) v[j] = x[row * a.ldx + c];
    }
    const u32 keep = a.drop.threshold ? unit_keep_bits<false>(a.drop, (uint64_t)row, col0, lane) : 0xFFu;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t c = col0 + lane_col<false>(lane, j);
      if (c < a.cols) y[row * a.ldy + c] = from_float<T>((keep >> j) & 1u ? to_float(v[j]) * a.drop.scale : 0.0f);
    }
  }
}

template <typename T>
int launch_dropout(const DropoutArgs& a, bool vec, int sms, cudaStream_t s) {
  const int64_t tasks = vec ? (a.rows * (a.cols >> 3) + kDropThreads - 1) / kDropThreads
                            : (a.rows * ((a.cols + 255) >> 8) + kDropThreads / 32 - 1) / (kDropThreads / 32);
  const int64_t most = (int64_t)sms * 8;
  const int blocks = (int)(tasks < most ? tasks : most);
  if (vec) k_dropout_vec<T><<<blocks, kDropThreads, 0, s>>>(a);
  else k_dropout_any<T><<<blocks, kDropThreads, 0, s>>>(a);
  return train_rc(cudaGetLastError());
}

// ---- a row in registers ----------------------------------------------------------------------------------------------
// A warp's share of a row: U units of 256 columns, as they lie in memory (16-bit types stay packed until used).
template <typename T, bool VEC, int U>
struct RowShare {
  Eight<T> v[U];
  __device__ __forceinline__ void load(const T* row, int64_t col0, int64_t cols, int lane) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t c0 = col0 + u * 256;
      if (VEC) {
        if (c0 + lane * 8 < cols) v[u].load(row + c0 + lane * 8);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int64_t c = c0 + lane_col<false>(lane, j);
          if (c < cols) reinterpret_cast<T*>(v[u].w)[j] = row[c];
        }
      }
    }
  }
  __device__ __forceinline__ void store(T* row, int64_t col0, int64_t cols, int lane) const {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t c0 = col0 + u * 256;
      if (VEC) {
        if (c0 + lane * 8 < cols) v[u].store(row + c0 + lane * 8);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int64_t c = c0 + lane_col<false>(lane, j);
          if (c < cols) row[c] = reinterpret_cast<const T*>(v[u].w)[j];
        }
      }
    }
  }
};

template <bool VEC> __device__ __forceinline__ bool has_col(int64_t col0, int u, int lane, int j, int64_t cols) {
  return col0 + u * 256 + (VEC ? lane * 8 : lane_col<false>(lane, j)) < cols;
}

// The weight vectors in shared memory, brought by 4-byte asynchronous copies (a view into a flat parameter vector is
// aligned no better) while the first row is on its way.  VEC lanes read their eight columns as two 16-byte words; each
// half of a unit is stored contiguously over the lanes so that these reads meet no bank twice.
template <bool VEC> __device__ __forceinline__ int weight_place(int c) {
  return VEC ? (c & ~255) + ((c >> 2) & 1) * 128 + ((c >> 3) & 31) * 4 + (c & 3) : c;
}
template <bool VEC> __device__ __forceinline__ void fetch_vector(float* to, const float* from, int cols) {
  for (int c = threadIdx.x; c < cols; c += blockDim.x) {
    float* dst = to + weight_place<VEC>(c);
    if (from) {
      const u32 at = (u32)__cvta_generic_to_shared(dst);
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(at), "l"(from + c) : "memory");
    } else {
      *dst = 0.0f;
    }
  }
}
__device__ __forceinline__ void fetched() {
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
}
template <bool VEC> __device__ __forceinline__ void read_vector(float (&out)[8], const float* from, int64_t col0, int lane) {
  if (VEC) {
    const float4 lo = *reinterpret_cast<const float4*>(from + col0 + lane * 4);
    const float4 hi = *reinterpret_cast<const float4*>(from + col0 + 128 + lane * 4);
    out[0] = lo.x; out[1] = lo.y; out[2] = lo.z; out[3] = lo.w;
    out[4] = hi.x; out[5] = hi.y; out[6] = hi.z; out[7] = hi.w;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) out[j] = from[col0 + lane_col<false>(lane, j)];
  }
}

// The sum over a row of what each lane holds: over the warp, and over the block where the whole block has one row.
// `slot` is 32 floats of shared memory that no warp may still be reading from an earlier call.
template <bool MULTI> __device__ __forceinline__ float row_sum(float v, float* slot) {
  v = warp_sum(v);
  if (MULTI) {
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0f;
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) v += slot[w];
  }
  return v;
}

// ---- layer norm, forward ---------------------------------------------------------------------------------------------
struct NormArgs {
  const void *x, *residual;
  const float *weight, *bias;
  void *y, *h;
  float *mean, *rstd;
  int64_t ldx, ldr, ldy, ldh, rows;
  int cols;
  float eps;
  Drop drop;
};

constexpr int kNormWarps = 4;  // rows of a block, one a warp, where a warp holds a whole row

// One warp per row (MULTI false), or one block per row.  Mean and variance are taken in two passes over the registers:
// the variance of centred values loses nothing when the mean is large beside the deviation.
template <typename T, typename S, bool VEC, int U, bool MULTI>
__global__ void __launch_bounds__(MULTI ? 512 : 32 * kNormWarps) k_norm(const NormArgs a) {
  extern __shared__ __align__(16) float smem[];
  __shared__ float slots[4][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t col0 = MULTI ? (int64_t)warp * (U * 256) : 0;
  const int padded = (a.cols + 255) & ~255;
  float *weight = smem, *bias = smem + padded;
  fetch_vector<VEC>(weight, a.weight, a.cols);
  fetch_vector<VEC>(bias, a.bias, a.cols);
  const int64_t step = (int64_t)gridDim.x * (MULTI ? 1 : kNormWarps);
  int64_t row = MULTI ? blockIdx.x : (int64_t)blockIdx.x * kNormWarps + warp;
  const float inv = 1.0f / (float)a.cols;
  bool first = true;
  for (int turn = 0; first || row < a.rows; row += step, turn ^= 2) {
    const bool real = row < a.rows;
    float f[U][8];
    float mean = 0.0f, rstd = 0.0f;
    if (real || MULTI) {  // a block has one row for all its warps: real is the same for them
      RowShare<T, VEC, U> x;
      RowShare<S, VEC, U> r;
      if (real) x.load(static_cast<const T*>(a.x) + row * a.ldx, col0, a.cols, lane);
      if (real && a.residual) r.load(static_cast<const S*>(a.residual) + row * a.ldr, col0, a.cols, lane);
      float sum = 0.0f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const u32 keep = a.drop.threshold ? unit_keep_bits<VEC>(a.drop, (uint64_t)row, col0 + u * 256, lane) : 0xFFu;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float v = (keep >> j) & 1u ? x.v[u].get(j) * a.drop.scale : 0.0f;
          if (a.residual) v += r.v[u].get(j);
          f[u][j] = real && has_col<VEC>(col0, u, lane, j, a.cols) ? v : 0.0f;
          sum += f[u][j];
        }
      }
      mean = row_sum<MULTI>(sum, slots[turn]) / (float)a.cols;  // a division: the mean of equal values is exact more often
      float square = 0.0f;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float c = f[u][j] - mean;
          if (has_col<VEC>(col0, u, lane, j, a.cols)) square += c * c;
        }
      rstd = 1.0f / sqrtf(row_sum<MULTI>(square, slots[turn + 1]) * inv + a.eps);
    }
    if (first) {
      fetched();
      first = false;
    }
    if (!real) continue;
    if (lane == 0 && (!MULTI || warp == 0)) {
      a.mean[row] = mean;
      a.rstd[row] = rstd;
    }
    if (a.h) {
      RowShare<S, VEC, U> h;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j) h.v[u].set(j, f[u][j]);
      h.store(static_cast<S*>(a.h) + row * a.ldh, col0, a.cols, lane);
    }
    RowShare<T, VEC, U> y;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float w[8], b[8];
      if (col0 + u * 256 < padded) {
        read_vector<VEC>(w, weight, col0 + u * 256, lane);
        read_vector<VEC>(b, bias, col0 + u * 256, lane);
#pragma unroll
        for (int j = 0; j < 8; ++j) y.v[u].set(j, (f[u][j] - mean) * rstd * w[j] + b[j]);
      }
    }
    y.store(static_cast<T*>(a.y) + row * a.ldy, col0, a.cols, lane);
  }
}

// ---- layer norm, backward --------------------------------------------------------------------------------------------
struct NormBackArgs {
  const void *dy, *h, *dh;
  const float *mean, *rstd, *weight;
  void *dx, *dres;
  int64_t ld_dy, ldh, ld_dh, ld_dx, ld_dres, rows, rows_per_block;
  int cols, groups;
  const int64_t* offsets;  // NULL: one group of all rows
  float* partial;          // [blocks + groups][2][padded cols], or NULL: no weight gradients
  Drop drop;
};

__device__ __forceinline__ int64_t offset_at(const int64_t* offsets, int g, int64_t rows) {
  if (!offsets) return g ? rows : 0;
  const int64_t v = offsets[g];
  return v < 0 ? 0 : v > rows ? rows : v;
}

// How many of offsets[1 .. groups] are at most `row`: the group that holds it, if the offsets ascend.  One load for
// every 32 groups, by the whole warp.
__device__ __forceinline__ int group_of(const int64_t* offsets, int groups, int64_t row, int64_t rows, int lane) {
  int n = 0;
  for (int g0 = 0; g0 < groups; g0 += 32) {
    const bool past = g0 + lane < groups && offset_at(offsets, g0 + lane + 1, rows) <= row;
    n += __popc(__ballot_sync(kAll, past));
  }
  return n;
}

// A block takes a contiguous range of rows, so that its warps can keep the sums of the weight gradients in registers;
// where the range meets the end of a group the sums so far go to the slot (block + group) of the partial sums.  With
// ascending groups no two blocks share a slot: a later block's groups are not lower, so block + group only grows.
template <typename T, typename S, bool VEC, int U, bool MULTI>
__global__ void __launch_bounds__(MULTI ? 512 : 32 * kNormWarps) k_norm_back(const NormBackArgs a) {
  extern __shared__ __align__(16) float smem[];
  __shared__ float slots[4][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t col0 = MULTI ? (int64_t)warp * (U * 256) : 0;
  const int padded = (a.cols + 255) & ~255;
  float *weight = smem, *joint = smem + padded;  // joint: 2 * padded floats, only without MULTI
  fetch_vector<VEC>(weight, a.weight, a.cols);
  const int64_t r0 = blockIdx.x * a.rows_per_block;
  const int64_t r1 = r0 + a.rows_per_block < a.rows ? r0 + a.rows_per_block : a.rows;
  const float inv = 1.0f / (float)a.cols;
  int g = a.partial ? group_of(a.offsets, a.groups, r0, a.rows, lane) : 0;
  fetched();
  int turn = 0;
  for (int64_t at = r0; at < r1;) {
    // rows [at, end) belong to one group, or to none
    int64_t end = r1;
    bool counted = false;
    if (a.partial && g < a.groups) {
      const int64_t lo = offset_at(a.offsets, g, a.rows), hi = offset_at(a.offsets, g + 1, a.rows);
      if (at < lo) {
        end = lo < r1 ? lo : r1;
      } else if (at < hi) {
        end = hi < r1 ? hi : r1;
        counted = true;
      } else {
        ++g;
        continue;
      }
    }
    float dw[U][8], db[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) dw[u][j] = db[u][j] = 0.0f;
    for (int64_t row = MULTI ? at : at + warp; row < end; row += MULTI ? 1 : kNormWarps, turn ^= 2) {
      RowShare<T, VEC, U> dy;
      RowShare<S, VEC, U> h, dh;
      dy.load(static_cast<const T*>(a.dy) + row * a.ld_dy, col0, a.cols, lane);
      h.load(static_cast<const S*>(a.h) + row * a.ldh, col0, a.cols, lane);
      if (a.dh) dh.load(static_cast<const S*>(a.dh) + row * a.ld_dh, col0, a.cols, lane);
      const float mean = a.mean[row], rstd = a.rstd[row];
      float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float w[8];
        if (col0 + u * 256 < padded) read_vector<VEC>(w, weight, col0 + u * 256, lane);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (has_col<VEC>(col0, u, lane, j, a.cols)) {
            const float d = dy.v[u].get(j), n = (h.v[u].get(j) - mean) * rstd, p = d * w[j];
            s1 += p;
            s2 += p * n;
            dw[u][j] += d * n;
            db[u][j] += d;
          }
        }
      }
      const float m1 = row_sum<MULTI>(s1, slots[turn]) * inv, m2 = row_sum<MULTI>(s2, slots[turn + 1]) * inv;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float w[8];
        if (col0 + u * 256 < padded) read_vector<VEC>(w, weight, col0 + u * 256, lane);
        const u32 keep = a.drop.threshold ? unit_keep_bits<VEC>(a.drop, (uint64_t)row, col0 + u * 256, lane) : 0xFFu;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float n = (h.v[u].get(j) - mean) * rstd;
          float v = (dy.v[u].get(j) * w[j] - m1 - n * m2) * rstd;
          if (a.dh) v += dh.v[u].get(j);
          h.v[u].set(j, v);
          dy.v[u].set(j, (keep >> j) & 1u ? v * a.drop.scale : 0.0f);
        }
      }
      dy.store(static_cast<T*>(a.dx) + row * a.ld_dx, col0, a.cols, lane);
      if (a.dres) h.store(static_cast<S*>(a.dres) + row * a.ld_dres, col0, a.cols, lane);
    }
    if (counted) {
      float* out = a.partial + (int64_t)(blockIdx.x + g) * 2 * padded;
      if (MULTI) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int64_t c = col0 + u * 256 + lane_col<VEC>(lane, j);
            if (c < a.cols) {
              out[c] = dw[u][j];
              out[padded + c] = db[u][j];
            }
          }
      } else {  // the warps add theirs one after the other, so that the order is fixed
        for (int w = 0; w < kNormWarps; ++w) {
          if (warp == w) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const int c = u * 256 + j * 32 + lane;  // any place will do that a lane finds again
                if (c < padded) {
                  joint[c] = w ? joint[c] + dw[u][j] : dw[u][j];
                  joint[padded + c] = w ? joint[padded + c] + db[u][j] : db[u][j];
                }
              }
          }
          __syncthreads();
        }
        for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
          const int e = c & 255, place = VEC ? (c & ~255) + (e & 7) * 32 + (e >> 3) : c;
          out[c] = joint[place];
          out[padded + c] = joint[padded + place];
        }
        __syncthreads();
      }
      ++g;
    }
    at = end;
  }
}

// The weight gradients: for each group the sum of its blocks' partial sums, eight runs of them side by side.
struct NormSumArgs {
  const float* partial;
  float *dweight, *dbias;
  int64_t ld_dweight, ld_dbias, rows, rows_per_block;
  int cols, accumulate;
  const int64_t* offsets;
};

__global__ void __launch_bounds__(256) k_norm_sum(const NormSumArgs a) {
  __shared__ float part[2][8][32];
  const int g = blockIdx.y, c = blockIdx.x * 32 + threadIdx.x, padded = (a.cols + 255) & ~255;
  const int64_t lo = offset_at(a.offsets, g, a.rows), hi = offset_at(a.offsets, g + 1, a.rows);
  float w = 0.0f, b = 0.0f;
  if (c < a.cols && lo < hi) {
    const int64_t last = (hi - 1) / a.rows_per_block;
    for (int64_t block = lo / a.rows_per_block + threadIdx.y; block <= last; block += 8) {
      const float* p = a.partial + (block + g) * 2 * padded;
      w += p[c];
      b += p[padded + c];
    }
  }
  part[0][threadIdx.y][threadIdx.x] = w;
  part[1][threadIdx.y][threadIdx.x] = b;
  __syncthreads();
  if (threadIdx.y < 2 && c < a.cols) {
    float* out = threadIdx.y ? a.dbias : a.dweight;
    if (!out) return;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += part[threadIdx.y][i][threadIdx.x];
    out += g * (threadIdx.y ? a.ld_dbias : a.ld_dweight) + c;
    *out = a.accumulate ? *out + s : s;
  }
}

// ---- choice of the variant -------------------------------------------------------------------------------------------
// A warp holds at most `most` units of a row; a wider row is shared by as many warps as that takes.
struct Share { int units, warps; };
inline Share share_of(int cols, int most) {
  const int n = (cols + 255) / 256, warps = (n + most - 1) / most;
  return {(n + warps - 1) / warps, warps};
}

template <typename K> bool ready(K kernel, size_t smem) {
  return smem <= 48 * 1024 || cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) == cudaSuccess;
}

template <typename T, typename S, bool VEC, int U, bool MULTI>
int launch_norm(const NormArgs& a, int warps, int sms, cudaStream_t s) {
  const size_t smem = 2 * sizeof(float) * ((a.cols + 255) & ~255);
  auto* k = k_norm<T, S, VEC, U, MULTI>;
  if (!ready(k, smem)) return train_rc(cudaGetLastError());
  const int threads = 32 * (MULTI ? warps : kNormWarps), per_block = MULTI ? 1 : kNormWarps;
  const int64_t tasks = (a.rows + per_block - 1) / per_block, most = (int64_t)sms * (2048 / threads);
  k<<<(int)(tasks < most ? tasks : most), threads, smem, s>>>(a);
  return train_rc(cudaGetLastError());
}

template <typename T, typename S, bool VEC>
int launch_norm_units(const NormArgs& a, int sms, cudaStream_t s) {
  const Share sh = share_of(a.cols, 4);
  if (sh.warps > 1) return sh.units == 3 ? launch_norm<T, S, VEC, 3, true>(a, sh.warps, sms, s) : launch_norm<T, S, VEC, 4, true>(a, sh.warps, sms, s);
  switch (sh.units) {
    case 1: return launch_norm<T, S, VEC, 1, false>(a, 1, sms, s);
    case 2: return launch_norm<T, S, VEC, 2, false>(a, 1, sms, s);
    case 3: return launch_norm<T, S, VEC, 3, false>(a, 1, sms, s);
    default: return launch_norm<T, S, VEC, 4, false>(a, 1, sms, s);
  }
}

// Rows of a block of the backward pass and the number of blocks: enough blocks to fill the machine, but no fewer than
// four rows a warp where there are that many, since every block leaves a row of partial sums behind.
constexpr int kBackBlocksPerSm = 4;
constexpr int kMostSms = 160;  // for the workspace's size, which is asked for without a device
inline int64_t back_rows_per_block(int64_t rows, int warps_per_row, int sms) {
  const int64_t parallel = warps_per_row > 1 ? 1 : kNormWarps;
  const int64_t most = (int64_t)(sms < kMostSms ? sms : kMostSms) * kBackBlocksPerSm;
  int64_t per = (rows + most - 1) / most;
  per = (per + parallel - 1) / parallel * parallel;
  return per < parallel ? parallel : per;
}

template <typename T, typename S, bool VEC, int U, bool MULTI>
int launch_norm_back(const NormBackArgs& a, int warps, cudaStream_t s) {
  const size_t smem = (MULTI ? 1 : 3) * sizeof(float) * ((a.cols + 255) & ~255);
  auto* k = k_norm_back<T, S, VEC, U, MULTI>;
  if (!ready(k, smem)) return train_rc(cudaGetLastError());
  const int64_t blocks = (a.rows + a.rows_per_block - 1) / a.rows_per_block;
  k<<<(int)blocks, 32 * (MULTI ? warps : kNormWarps), smem, s>>>(a);
  return train_rc(cudaGetLastError());
}

// The backward pass holds three arrays and two sums of a row: binary32 rows get half the units a warp, up to the
// sixteen warps of a block; only beyond 8,192 columns they get four after all, and the compiler keeps some in memory.
inline Share back_share(int cols, size_t size, size_t ssize) {
  return share_of(cols, size + ssize == 4 || cols > 16 * 2 * 256 ? 4 : 2);
}

template <typename T, typename S, bool VEC>
int launch_norm_back_units(const NormBackArgs& a, cudaStream_t s) {
  constexpr bool kShort = sizeof(T) + sizeof(S) == 4;
  const Share sh = back_share(a.cols, sizeof(T), sizeof(S));
  if (sh.warps > 1)
    return sh.units == 2 ? launch_norm_back<T, S, VEC, 2, true>(a, sh.warps, s)
           : kShort && sh.units == 3 ? launch_norm_back<T, S, VEC, kShort ? 3 : 4, true>(a, sh.warps, s)
                                     : launch_norm_back<T, S, VEC, 4, true>(a, sh.warps, s);
  switch (sh.units) {
    case 1: return launch_norm_back<T, S, VEC, 1, false>(a, 1, s);
    case 2: return launch_norm_back<T, S, VEC, 2, false>(a, 1, s);
    case 3: return launch_norm_back<T, S, VEC, kShort ? 3 : 2, false>(a, 1, s);  // more than two: 16-bit rows only
    default: return launch_norm_back<T, S, VEC, kShort ? 4 : 2, false>(a, 1, s);
  }
}

}  // namespace

extern "C" {

int regtopk_dropout(const void* x, int64_t ldx, void* y, int64_t ldy, int64_t rows, int64_t cols, int32_t type,
                    const regtopk_dropout_params* drop, void* cuda_stream) {
  DropoutArgs a;
  const size_t size = type_size(type);
  if (!size || !drop || rows < 0 || cols < 0 || cols > (int64_t)1 << 34 || !make_drop(drop, &a.drop)) return REGTOPK_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return REGTOPK_OK;
  if (!good_matrix(x, ldx, rows, cols, size) || !good_matrix(y, ldy, rows, cols, size)) return REGTOPK_ERR_INVALID_ARG;
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  a.x = x; a.y = y; a.ldx = ldx; a.ldy = ldy; a.rows = rows; a.cols = cols;
  const bool vec = cols % 8 == 0 && rows_aligned(x, ldx, size, rows) && rows_aligned(y, ldy, size, rows);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  switch (type) {
    case REGTOPK_TYPE_F32: return launch_dropout<float>(a, vec, sms, s);
    case REGTOPK_TYPE_BF16: return launch_dropout<__nv_bfloat16>(a, vec, sms, s);
    default: return launch_dropout<__half>(a, vec, sms, s);
  }
}

#define REGTOPK_BY_TYPE(call)                                                                            \
  if (type == REGTOPK_TYPE_F32) return vec ? call(float, float, true) : call(float, float, false);        \
  if (type == REGTOPK_TYPE_BF16 && stream_type == type)                                                   \
    return vec ? call(__nv_bfloat16, __nv_bfloat16, true) : call(__nv_bfloat16, __nv_bfloat16, false);    \
  if (type == REGTOPK_TYPE_BF16) return vec ? call(__nv_bfloat16, float, true) : call(__nv_bfloat16, float, false); \
  if (stream_type == type) return vec ? call(__half, __half, true) : call(__half, __half, false);         \
  return vec ? call(__half, float, true) : call(__half, float, false)

int regtopk_layer_norm(const void* x, int64_t ldx, const void* residual, int64_t ld_residual, const float* weight,
                       const float* bias, float eps, void* y, int64_t ldy, void* h, int64_t ldh, float* mean,
                       float* rstd, int64_t rows, int64_t cols, int32_t type, int32_t stream_type,
                       const regtopk_dropout_params* drop, void* cuda_stream) {
  NormArgs a;
  const size_t size = type_size(type), ssize = type_size(stream_type);
  if (!size || !ssize || (stream_type != type && stream_type != REGTOPK_TYPE_F32) || rows < 0 || cols < 1 ||
      !(eps >= 0.0f && eps <= 3.4e38f) || !make_drop(drop, &a.drop)) return REGTOPK_ERR_INVALID_ARG;
  if (cols > REGTOPK_NORM_MAX_COLS) return REGTOPK_ERR_TOO_LARGE;
  if (rows == 0) return REGTOPK_OK;
  if (!good_matrix(x, ldx, rows, cols, size) || !good_matrix(y, ldy, rows, cols, size) ||
      (residual && !good_matrix(residual, ld_residual, rows, cols, ssize)) || (h && !good_matrix(h, ldh, rows, cols, ssize)) ||
      !good_matrix(weight, cols, 1, cols, 4) || !good_matrix(mean, 1, 1, 1, 4) || !good_matrix(rstd, 1, 1, 1, 4) ||
      (uintptr_t)bias % 4) return REGTOPK_ERR_INVALID_ARG;
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  a.x = x; a.residual = residual; a.weight = weight; a.bias = bias; a.y = y; a.h = h; a.mean = mean; a.rstd = rstd;
  a.ldx = ldx; a.ldr = ld_residual; a.ldy = ldy; a.ldh = ldh; a.rows = rows; a.cols = (int)cols; a.eps = eps;
  const bool vec = cols % 8 == 0 && rows_aligned(x, ldx, size, rows) && rows_aligned(y, ldy, size, rows) &&
                   rows_aligned(residual, ld_residual, ssize, rows) && rows_aligned(h, ldh, ssize, rows);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
#define REGTOPK_NORM(T, S, V) launch_norm_units<T, S, V>(a, sms, s)
  REGTOPK_BY_TYPE(REGTOPK_NORM);
#undef REGTOPK_NORM
}

size_t regtopk_layer_norm_backward_workspace_bytes(int64_t rows, int64_t cols, int32_t groups) {
  if (rows < 0 || cols < 1 || cols > REGTOPK_NORM_MAX_COLS || groups < 1) return 0;
  const int64_t most = (int64_t)kMostSms * kBackBlocksPerSm;
  return ((rows < most ? rows : most) + (size_t)groups) * 2 * ((cols + 255) & ~255) * sizeof(float);
}

int regtopk_layer_norm_backward(const void* dy, int64_t ld_dy, const void* h, int64_t ldh, const float* mean,
                                const float* rstd, const float* weight, const void* dh, int64_t ld_dh, void* dx,
                                int64_t ld_dx, void* dresidual, int64_t ld_dresidual, float* dweight,
                                int64_t ld_dweight, float* dbias, int64_t ld_dbias, const int64_t* offsets,
                                int32_t groups, int32_t accumulate, int64_t rows, int64_t cols, int32_t type,
                                int32_t stream_type, const regtopk_dropout_params* drop, void* workspace,
                                size_t workspace_bytes, void* cuda_stream) {
  NormBackArgs a;
  const size_t size = type_size(type), ssize = type_size(stream_type);
  const bool sums = dweight || dbias;
  if (!size || !ssize || (stream_type != type && stream_type != REGTOPK_TYPE_F32) || rows < 0 || cols < 1 || groups < 1 ||
      groups > 65535 || (!offsets && groups != 1) || (uintptr_t)offsets % 8 || !make_drop(drop, &a.drop)) return REGTOPK_ERR_INVALID_ARG;
  if (cols > REGTOPK_NORM_MAX_COLS) return REGTOPK_ERR_TOO_LARGE;
  if ((dweight && !good_matrix(dweight, ld_dweight, groups, cols, 4)) || (dbias && !good_matrix(dbias, ld_dbias, groups, cols, 4)))
    return REGTOPK_ERR_INVALID_ARG;
  if (rows > 0 && (!good_matrix(dy, ld_dy, rows, cols, size) || !good_matrix(h, ldh, rows, cols, ssize) ||
                   !good_matrix(dx, ld_dx, rows, cols, size) || (dh && !good_matrix(dh, ld_dh, rows, cols, ssize)) ||
                   (dresidual && !good_matrix(dresidual, ld_dresidual, rows, cols, ssize)) ||
                   !good_matrix(weight, cols, 1, cols, 4) || !good_matrix(mean, 1, 1, 1, 4) || !good_matrix(rstd, 1, 1, 1, 4)))
    return REGTOPK_ERR_INVALID_ARG;
  if (sums && rows > 0) {
    if (!workspace || (uintptr_t)workspace % 16) return REGTOPK_ERR_INVALID_ARG;
    if (workspace_bytes < regtopk_layer_norm_backward_workspace_bytes(rows, cols, groups)) return REGTOPK_ERR_WORKSPACE_TOO_SMALL;
  }
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  a.dy = dy; a.h = h; a.dh = dh; a.mean = mean; a.rstd = rstd; a.weight = weight; a.dx = dx; a.dres = dresidual;
  a.ld_dy = ld_dy; a.ldh = ldh; a.ld_dh = ld_dh; a.ld_dx = ld_dx; a.ld_dres = ld_dresidual; a.rows = rows; a.cols = (int)cols;
  a.groups = groups; a.offsets = offsets; a.partial = sums ? static_cast<float*>(workspace) : nullptr;
  const Share sh = back_share((int)cols, size, ssize);
  a.rows_per_block = back_rows_per_block(rows, sh.warps, sms);
  if (rows > 0) {
    const bool vec = cols % 8 == 0 && rows_aligned(dy, ld_dy, size, rows) && rows_aligned(h, ldh, ssize, rows) &&
                     rows_aligned(dh, ld_dh, ssize, rows) && rows_aligned(dx, ld_dx, size, rows) &&
                     rows_aligned(dresidual, ld_dresidual, ssize, rows);
    auto launch = [&]() -> int {
#define REGTOPK_NORM_BACK(T, S, V) launch_norm_back_units<T, S, V>(a, s)
      REGTOPK_BY_TYPE(REGTOPK_NORM_BACK);
#undef REGTOPK_NORM_BACK
    };
    const int rc = launch();
    if (rc != REGTOPK_OK) return rc;
  }
  if (sums) {
    NormSumArgs n;
    n.partial = a.partial; n.dweight = dweight; n.dbias = dbias; n.ld_dweight = ld_dweight; n.ld_dbias = ld_dbias;
    n.rows = rows; n.rows_per_block = a.rows_per_block; n.cols = (int)cols; n.accumulate = accumulate; n.offsets = offsets;
    k_norm_sum<<<dim3((unsigned)((cols + 31) / 32), (unsigned)groups), dim3(32, 8), 0, s>>>(n);
    return train_rc(cudaGetLastError());
  }
  return REGTOPK_OK;
}

}  // extern "C"
