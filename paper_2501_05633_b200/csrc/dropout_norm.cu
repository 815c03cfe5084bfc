// Dropout and layer norm with their gradients (include/regtopk_train.h).
//
// All of them have memory traffic for their floor: a few operations per element and one read and one write of each array.
// So each kernel reads every input once, keeps many copies under way, and draws the dropout mask again wherever it is
// needed instead of storing it (one Philox call for eight columns costs less issue time than a byte of mask costs
// bandwidth).  Dropout reaches that floor.  The norms spend 40 to 46 instructions of a lane on a value at 16 to 24 warps an SM:
// little over half of the issue slots and of the memory's bandwidth are in use, and it is the latency between the two, with too few
// warps to hide it, that binds them.

#include "norm_rows.cuh"

namespace {

// ---- dropout -------------------------------------------------------------------------------------------------------
struct DropoutArgs {
  const void* x;
  void* y;
  int64_t ldx, ldy, rows, cols;
  u32 groups, total, magic, shift;  // k_dropout_vec: groups of eight columns in a row and in all; division by the former
  Drop drop;
};

constexpr int kDropThreads = 256;
constexpr int kDropStep = 2;  // loads under way per thread

// Aligned rows of a multiple of eight columns, fewer than 2^31 groups of eight: a thread takes kDropStep groups at a
// time.  The row of a group is found by a multiplication (Granlund and Montgomery 1994): with 2^(s-1) < d <= 2^s and
// magic = floor(2^(31+s) / d) + 1, which has 32 bits, floor(n / d) = floor(2n magic / 2^(32+s)) for every n < 2^31.
template <typename T>
__global__ void __launch_bounds__(kDropThreads) k_dropout_vec(const DropoutArgs a) {
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.y);
  const u32 first = blockIdx.x * (kDropThreads * kDropStep);
  Eight<T> v[kDropStep];
  u32 row[kDropStep], group[kDropStep];
  begin_after_predecessor();
#pragma unroll
  for (int i = 0; i < kDropStep; ++i) {
    const u32 at = first + i * kDropThreads + threadIdx.x;
    row[i] = __umulhi(2 * at, a.magic) >> a.shift;
    group[i] = at - row[i] * a.groups;
    if (at < a.total) v[i].fetch(x + (row[i] * a.ldx + (uint64_t)group[i] * 8));
  }
#pragma unroll
  for (int i = 0; i < kDropStep; ++i) {
    const u32 at = first + i * kDropThreads + threadIdx.x;
    if (a.drop.threshold) {
      Octet f;
      v[i].get(f);
      Numbers(a.drop, row[i], group[i]).drop(f, a.drop);
      v[i].put(f);
    }
    if (at < a.total) v[i].store(y + (row[i] * a.ldy + (uint64_t)group[i] * 8));
  }
}

// Any other layout: a warp takes 256 columns of a row, element by element (8,192 x 2,047 bfloat16: 25 us, where the layout
// with 2,048 columns takes 13.6 us in the kernel above; aligned words shifted together took 42 us).
template <typename T>
__global__ void __launch_bounds__(kDropThreads) k_dropout_any(const DropoutArgs a) {
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.y);
  const int lane = threadIdx.x & 31;
  const int64_t units = (a.cols + 255) >> 8, total = a.rows * units;
  begin_after_predecessor();
  const int64_t step = (int64_t)gridDim.x * (kDropThreads / 32);
  for (int64_t at = (int64_t)blockIdx.x * (kDropThreads / 32) + (threadIdx.x >> 5); at < total; at += step) {
    const int64_t row = total >> 32 ? at / units : (u32)at / (u32)units, col0 = (at - row * units) << 8;
    Octet f;
    read_eight<T, false, false>(f, x + row * a.ldx, col0, lane, a.cols);
    if (a.drop.threshold) drop_unit<false>(f, a.drop, (uint64_t)row, col0, lane);
    store_eight<T, false>(f, y + row * a.ldy, col0, lane, a.cols);
  }
}

template <typename T>
int launch_dropout(DropoutArgs& a, bool vec, int sms, cudaStream_t s) {
  const int64_t groups = a.cols >> 3;
  if (vec && a.rows * groups < (int64_t)1 << 31) {
    int s31 = 0;
    while (((int64_t)1 << s31) < groups) ++s31;
    a.groups = (u32)groups;
    a.total = (u32)(a.rows * groups);
    a.magic = (u32)(((uint64_t)1 << (31 + s31)) / (uint64_t)groups + 1);
    a.shift = (u32)s31;
    return start(k_dropout_vec<T>, (a.total + kDropThreads * kDropStep - 1) / (kDropThreads * kDropStep), kDropThreads, 0, s, a);
  } else {
    const int64_t tasks = (a.rows * ((a.cols + 255) >> 8) + kDropThreads / 32 - 1) / (kDropThreads / 32), most = (int64_t)sms * 8;
    return start(k_dropout_any<T>, (unsigned)(tasks < most ? tasks : most), kDropThreads, 0, s, a);
  }
}

// ---- layer norm, forward ---------------------------------------------------------------------------------------------
struct NormArgs {
  Source source[3];  // x, residual
  const float *weight, *bias;
  void *y, *h;
  float *mean, *rstd;
  int64_t ldy, ldh, rows;
  int cols, wide;
  float eps;
  Drop drop;
  RingShape ring;
};

// Mean and sum of squared deviations come from the registers in two passes within a warp and are then combined over the
// team by the rule for joining two samples (Chan, Golub, LeVeque 1979): nothing is lost when the mean is large beside the
// deviation, and one exchange a row is enough.
// RING false: a team has a few rows at most (plan_of says how many) and reads them, and the vectors for each, where they are.
// 32,768 rows of 1,024 bfloat16 columns with dropout beside a binary32 stream, 403 MB: 70 to 77 us, 5.2 to 5.8 TB/s, with 60 %
// of the issue slots busy.
template <typename T, typename S, bool VEC, int U, bool RING>
__global__ void __maxnreg__(U <= 2 ? 80 : 128) k_norm(const __grid_constant__ NormArgs a) {
  extern __shared__ __align__(16) char smem[];
  __shared__ Common common;
  const Team t(a.ring.warps, U);
  begin_after_predecessor();
  float *weight = reinterpret_cast<float*>(smem), *bias = weight + padded(a.cols);
  const int64_t first = (int64_t)blockIdx.x * a.ring.teams + t.index, step = (int64_t)gridDim.x * a.ring.teams;
  Ring<true> ring = make_ring<RING, true>(common, a.ring, a.source, reinterpret_cast<char*>(bias + padded(a.cols)), t, first, step, a.rows);
  if (RING) {
    fetch_vector<VEC>(weight, a.weight, a.cols);
    fetch_vector<VEC>(bias, a.bias, a.cols);
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
  }
  // columns of every warp but the last, and of the last; of this warp
  const float full = U * 256, last = (float)(a.cols - (t.warps - 1) * U * 256), own = t.warp == t.warps - 1 ? last : full;
  const float cols = (float)a.cols, per_col = 1.0f / cols, per_own = 1.0f / own;
  T* y = static_cast<T*>(a.y) + first * a.ldy;
  S* sum_out = static_cast<S*>(a.h) + first * a.ldh;
  const int64_t y_leap = step * a.ldy, h_leap = step * a.ldh;
  u32 turn = 0;
  for (int64_t row = first; row < a.rows; row += step, turn ^= 1, y += y_leap, sum_out += h_leap) {
    if (RING) ring.await(t.leads());
    Octet f[U];
    float2 sum = both(0.0f), square = both(0.0f);
    const T* x = ring.row_of<T, VEC, RING>(row, 0);
    const S* residual = ring.row_of<S, VEC, RING>(row, 1);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c0 = t.col0 + u * 256;
      read_eight<T, VEC, RING>(f[u], x, c0, t.lane, a.cols);
      if (a.drop.threshold) drop_unit<VEC>(f[u], a.drop, (uint64_t)row, c0, t.lane);
      if (a.ring.row_bytes[1]) {
        Octet r;
        read_eight<S, VEC, RING>(r, residual, c0, t.lane, a.cols);
#pragma unroll
        for (int i = 0; i < 4; ++i) f[u][i] = add2(f[u][i], r[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) sum = add2(sum, f[u][i]);  // zeros past the end
    }
    float mean = quotient(warp_sum(sum.x + sum.y), own, per_own);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c0 = t.col0 + u * 256;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float2 c = add2(f[u][i], both(-mean));
        if (VEC ? c0 + t.lane * 8 >= a.cols : c0 + lane_col<false>(t.lane, 2 * i) >= a.cols) c.x = 0.0f;
        if (VEC ? c0 + t.lane * 8 >= a.cols : c0 + lane_col<false>(t.lane, 2 * i + 1) >= a.cols) c.y = 0.0f;
        square = fma2(c, c, square);
      }
    }
    float spread = warp_sum(square.x + square.y);
    if (t.warps > 1 && t.lane == 0) common.exchange[turn][t.index * t.warps + t.warp] = make_float2(mean, spread);
    if (RING || t.warps > 1) t.sync();  // the row has been read by all
    if (RING) ring.pass(row, t.leads());
    if (t.warps > 1) {
      const float2* v = &common.exchange[turn][t.index * t.warps];
      const float2 end = v[t.warps - 1];
      mean = 0.0f;
      for (int i = 0; i < t.warps - 1; ++i) mean += v[i].x;
      mean = quotient(fmaf(full, mean, last * end.x), cols, per_col);
      spread = fmaf(last * (end.x - mean), end.x - mean, end.y);
      for (int i = 0; i < t.warps - 1; ++i) spread += fmaf(full * (v[i].x - mean), v[i].x - mean, v[i].y);
    }
    const float rstd = inverse_root(fmaf(spread, per_col, a.eps));
    if (t.leads()) {
      a.mean[row] = mean;
      a.rstd[row] = rstd;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c0 = t.col0 + u * 256;
      if (c0 >= a.cols) break;
      if (a.h) store_eight<S, VEC>(f[u], sum_out, c0, t.lane, a.cols);
      Octet w, b;
      if (RING) {
        read_vector<VEC>(w, weight, c0, t.lane);
        read_vector<VEC>(b, bias, c0, t.lane);
      } else {
        load_vector<VEC>(w, a.weight, a.wide, c0, t.lane, a.cols);
        load_vector<VEC>(b, a.bias, a.wide, c0, t.lane, a.cols);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) f[u][i] = fma2(mul2(add2(f[u][i], both(-mean)), both(rstd)), w[i], b[i]);
      store_eight<T, VEC>(f[u], y, c0, t.lane, a.cols);
    }
  }
}

// ---- layer norm, backward --------------------------------------------------------------------------------------------
struct NormBackArgs {
  Source source[3];  // dy, h, dh
  const float *mean, *rstd, *weight;
  void *dx, *dres;
  int64_t ld_dx, ld_dres, rows, block_rows;
  int cols, groups, wide;
  const int64_t* offsets;  // NULL: one group of all rows
  float* partial;          // [blocks + groups][2][cols], or NULL: no weight gradients
  Drop drop;
  RingShape ring;
};

// A block takes `block_rows` rows in a row, its teams one after the other in turn, and keeps the sums of the weight
// gradients in registers; where the range meets the end of a group the sums so far go to the slot (block + group) of
// the partial sums.  With ascending groups no two blocks share a slot: a later block's groups are not lower, so
// block + group only grows.
// 32,768 rows of 1,024 bfloat16 columns with dropout, 336 MB: 83 to 85 us with the sum after it, 4.0 TB/s.  58 % of the issue slots
// are busy with eight warps a block, whose 128 registers a thread leave no room for more of them.
template <typename T, typename S, bool VEC, int U, bool RING>
__global__ void __launch_bounds__(32 * kMostWarps, 1) k_norm_back(const __grid_constant__ NormBackArgs a) {
  extern __shared__ __align__(16) char smem[];
  __shared__ Common common;
  const Team t(a.ring.warps, U);
  begin_after_predecessor();
  float *weight = reinterpret_cast<float*>(smem), *joint = weight + padded(a.cols);  // joint: the teams' sums, if there are two or more
  const int64_t r0 = blockIdx.x * a.block_rows, r1 = min(a.rows, r0 + a.block_rows), first = r0 + t.index, step = a.ring.teams;
  Ring<false> ring = make_ring<RING, false>(common, a.ring, a.source, reinterpret_cast<char*>(joint + (a.ring.teams > 1 ? 2 * padded(a.cols) : 0)), t, first, step, r1);
  if (RING) fetch_vector<VEC>(weight, a.weight, a.cols);
  int g = a.partial ? group_of(a.offsets, a.groups, r0, a.rows, t.lane) : a.groups;
  float mean = 0.0f, rstd = 0.0f;
  if (first < r1) {
    mean = a.mean[first];
    rstd = a.rstd[first];
  }
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
    Octet dw[U], db[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) dw[u][i] = db[u][i] = both(0.0f);
    for (; row < end; row += step, turn ^= 1) {
      float next_mean = 0.0f, next_rstd = 0.0f;
      if (row + step < r1) {
        next_mean = a.mean[row + step];
        next_rstd = a.rstd[row + step];
      }
      if (RING) ring.await(t.leads());
      const T* dy = ring.row_of<T, VEC, RING>(row, 0);
      const S* h = ring.row_of<S, VEC, RING>(row, 1);
      float2 s1 = both(0.0f), s2 = both(0.0f);
      constexpr int kKept = RING ? 1 : U;  // without rings, what has been read stays in registers
      Octet kept_d[kKept], kept_v[kKept], kept_w[kKept];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c0 = t.col0 + u * 256;
        if (c0 >= a.cols) break;
        Octet &d = kept_d[u % kKept], &v = kept_v[u % kKept], &w = kept_w[u % kKept];
        read_eight<T, VEC, RING>(d, dy, c0, t.lane, a.cols);  // zeros past the end, so finite values add nothing there
        read_eight<S, VEC, RING>(v, h, c0, t.lane, a.cols, mean);
        if (RING) read_vector<VEC>(w, weight, c0, t.lane);
        else load_vector<VEC>(w, a.weight, a.wide, c0, t.lane, a.cols);
        // The difference first, which takes an instruction more than h rstd + (-mean rstd), 1 to 3 % of the time, but is exact
        // where the two are close: with a mean a thousand times the deviation dweight was off by 2e-5 of its largest value, now
        // as without a mean by 1e-7.  Past the end it is made 0: -mean there, times rstd, may be an infinity.
        const float centre = VEC && c0 + t.lane * 8 >= a.cols ? 0.0f : mean;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = add2(v[i], both(-centre));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 unit = mul2(v[i], both(rstd)), p = mul2(d[i], w[i]);
          s1 = add2(s1, p);
          s2 = fma2(p, unit, s2);
          dw[u][i] = fma2(d[i], unit, dw[u][i]);
          db[u][i] = add2(db[u][i], d[i]);
        }
      }
      float m1 = warp_sum(s1.x + s1.y), m2 = warp_sum(s2.x + s2.y);
      if (t.warps > 1) {
        if (t.lane == 0) common.exchange[turn][t.index * t.warps + t.warp] = make_float2(m1, m2);
        t.sync();
        const float2* v = &common.exchange[turn][t.index * t.warps];
        m1 = m2 = 0.0f;
        for (int i = 0; i < t.warps; ++i) {
          m1 += v[i].x;
          m2 += v[i].y;
        }
      }
      m1 *= inv;
      m2 *= inv;
      const float slope = -m2 * rstd;  // rstd (dy w - m1 - unit m2) = rstd (dy w - m1 + (h - mean) slope)
      if (RING) asm volatile("" ::: "memory");  // what follows is read from shared memory again: kept, it would not fit the registers
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c0 = t.col0 + u * 256;
        if (c0 >= a.cols) break;
        Octet &d = kept_d[u % kKept], &v = kept_v[u % kKept], &w = kept_w[u % kKept];
        if (RING) {
          read_eight<T, VEC, RING>(d, dy, c0, t.lane, a.cols);
          read_eight<S, VEC, RING>(v, h, c0, t.lane, a.cols);
          read_vector<VEC>(w, weight, c0, t.lane);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (RING) v[i] = add2(v[i], both(-mean));  // without rings what is kept is the difference
          d[i] = mul2(fma2(v[i], both(slope), fma2(d[i], w[i], both(-m1))), both(rstd));
        }
        if (a.ring.row_bytes[2]) {
          read_eight<S, VEC, RING>(v, ring.row_of<S, VEC, RING>(row, 2), c0, t.lane, a.cols);
#pragma unroll
          for (int i = 0; i < 4; ++i) d[i] = add2(d[i], v[i]);
        }
        if (a.dres) store_eight<S, VEC>(d, static_cast<S*>(a.dres) + row * a.ld_dres, c0, t.lane, a.cols);
        if (a.drop.threshold) drop_unit<VEC>(d, a.drop, (uint64_t)row, c0, t.lane);
        store_eight<T, VEC>(d, static_cast<T*>(a.dx) + row * a.ld_dx, c0, t.lane, a.cols);
      }
      if (RING || t.warps > 1) t.sync();  // the row has been read by all
      if (RING) ring.pass(row, t.leads());
      mean = next_mean;
      rstd = next_rstd;
    }
    if (counted) {
      float* out = a.partial + (int64_t)(blockIdx.x + g) * 2 * a.cols;
      if (a.ring.teams > 1) {  // the teams add theirs one after the other, so that the order is fixed
        for (int i = 0; i < a.ring.teams; ++i) {
          if (t.index == i) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
              const int c0 = t.col0 + u * 256;
              if (c0 >= a.cols) break;
              // any place will do that a lane finds again: pair k of the lane's eight lies at k * 64 + lane * 2
              float2 *w = reinterpret_cast<float2*>(joint + c0) + t.lane, *b = reinterpret_cast<float2*>(joint + padded(a.cols) + c0) + t.lane;
              if (i) {
                Octet ow, ob;
#pragma unroll
                for (int k = 0; k < 4; ++k) ow[k] = w[k * 32], ob[k] = b[k * 32];
#pragma unroll
                for (int k = 0; k < 4; ++k) dw[u][k] = add2(ow[k], dw[u][k]), db[u][k] = add2(ob[k], db[u][k]);
              }
#pragma unroll
              for (int k = 0; k < 4; ++k) w[k * 32] = dw[u][k], b[k * 32] = db[u][k];
            }
          }
          __syncthreads();
        }
        for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
          const int e = c & 255, lane = VEC ? e >> 3 : e & 31, j = VEC ? e & 7 : e >> 5, place = (c & ~255) + (j >> 1) * 64 + lane * 2 + (j & 1);
          out[c] = joint[place];
          out[a.cols + c] = joint[padded(a.cols) + place];
        }
        __syncthreads();
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int c = t.col0 + u * 256 + lane_col<VEC>(t.lane, j);
            if (c < a.cols) {
              out[c] = (j & 1) ? dw[u][j >> 1].y : dw[u][j >> 1].x;
              out[a.cols + c] = (j & 1) ? db[u][j >> 1].y : db[u][j >> 1].x;
            }
          }
      }
      ++g;
    }
    at = end;
  }
}

// The weight gradients: for each group the sum of its blocks' partial sums, kRuns runs of them side by side.  Always the
// same runs in the same order, so that the sums do not change from call to call.  Latency bounds it: 8 us for eight groups of
// 1,024 columns and 293 blocks, 2.4 MB, from memory.
struct NormSumArgs {
  const float* partial;
  float *dweight, *dbias;
  int64_t ld_dweight, ld_dbias, rows, block_rows;
  int cols, accumulate;
  const int64_t* offsets;
};

constexpr int kRuns = 16;
__global__ void __launch_bounds__(32 * kRuns) k_norm_sum(const NormSumArgs a) {
  __shared__ float part[2][kRuns][33];
  begin_after_predecessor();
  const int g = blockIdx.y, c = blockIdx.x * 32 + threadIdx.x;
  const int64_t lo = offset_at(a.offsets, g, a.rows), hi = offset_at(a.offsets, g + 1, a.rows);
  float w = 0.0f, b = 0.0f;
  if (c < a.cols && lo < hi) {
    const int64_t last = (hi - 1) / a.block_rows;
#pragma unroll 4
    for (int64_t block = lo / a.block_rows + threadIdx.y; block <= last; block += kRuns) {
      const float* p = a.partial + (block + g) * 2 * a.cols;
      w += p[c];
      b += p[a.cols + c];
    }
  }
  part[0][threadIdx.y][threadIdx.x] = w;
  part[1][threadIdx.y][threadIdx.x] = b;
  __syncthreads();
  // each warp adds the runs of some of the 64 sums, a lane a run
#pragma unroll
  for (int i = threadIdx.y; i < 64; i += kRuns) {
    const int which = i & 1, at = blockIdx.x * 32 + (i >> 1);
    const float s = warp_sum((int)threadIdx.x < kRuns ? part[which][threadIdx.x][i >> 1] : 0.0f);
    float* out = which ? a.dbias : a.dweight;
    if (threadIdx.x == 0 && out && at < a.cols) {
      out += g * (which ? a.ld_dbias : a.ld_dweight) + at;
      *out = a.accumulate ? *out + s : s;
    }
  }
}

// ---- launches --------------------------------------------------------------------------------------------------------
template <typename T, typename S, bool VEC, int U>
int launch_norm(const NormArgs& a, const Plan& p, int dev, int sms, cudaStream_t s) {
  const int64_t tasks = (a.rows + a.ring.teams - 1) / a.ring.teams, most = (int64_t)sms * p.blocks;
  const int blocks = (int)(tasks < most ? tasks : most);
  if (p.rings) {
    constexpr auto k = k_norm<T, S, VEC, U, true>;
    if (!allow_smem<k>(dev)) return train_rc(cudaGetLastError());
    return start(k, blocks, p.threads, p.smem, s, a);
  }
  return start(k_norm<T, S, VEC, U, false>, blocks, p.threads, 0, s, a);
}

template <typename T, typename S, bool VEC, int U>
int launch_norm_back(const NormBackArgs& a, const Plan& p, int dev, cudaStream_t s) {
  const int blocks = (int)((a.rows + a.block_rows - 1) / a.block_rows);
  if (p.rings) {
    constexpr auto k = k_norm_back<T, S, VEC, U, true>;
    if (!allow_smem<k>(dev)) return train_rc(cudaGetLastError());
    return start(k, blocks, p.threads, p.smem, s, a);
  }
  constexpr auto k = k_norm_back<T, S, VEC, U, false>;
  if (!allow_smem<k>(dev)) return train_rc(cudaGetLastError());
  return start(k, blocks, p.threads, p.smem, s, a);
}

}  // namespace

int regtopk_norm_gave_up(cudaStream_t s) { return gave_up(s); }

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

// `call` with the types, the layout and the units of a warp: TYPES is one of the five pairs of element and stream type.
#define REGTOPK_BY_UNITS(call, T, S, V) \
  (p.units == 1 ? call(T, S, V, 1) : p.units == 2 ? call(T, S, V, 2) : p.units == 3 ? call(T, S, V, 3) : call(T, S, V, 4))
#define REGTOPK_BY_LAYOUT(call, T, S) (vec ? REGTOPK_BY_UNITS(call, T, S, true) : REGTOPK_BY_UNITS(call, T, S, false))
#define REGTOPK_BY_TYPE(call)                                                              \
  (type == REGTOPK_TYPE_F32    ? REGTOPK_BY_LAYOUT(call, float, float)                     \
   : type == REGTOPK_TYPE_BF16 ? (stream_type == type ? REGTOPK_BY_LAYOUT(call, __nv_bfloat16, __nv_bfloat16) \
                                                      : REGTOPK_BY_LAYOUT(call, __nv_bfloat16, float))        \
   : stream_type == type       ? REGTOPK_BY_LAYOUT(call, __half, __half)                   \
                               : REGTOPK_BY_LAYOUT(call, __half, float))

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
  a.source[0] = {static_cast<const char*>(x), ldx * (int64_t)size};
  a.source[1] = {static_cast<const char*>(residual), ld_residual * (int64_t)ssize};
  a.source[2] = {nullptr, 0};
  a.weight = weight; a.bias = bias; a.y = y; a.h = h; a.mean = mean; a.rstd = rstd; a.ldy = ldy; a.ldh = ldh; a.rows = rows;
  a.cols = (int)cols; a.eps = eps; a.wide = (uintptr_t)weight % 16 == 0 && (uintptr_t)bias % 16 == 0;
  const bool vec = cols % 8 == 0 && rows_aligned(x, ldx, size, rows) && rows_aligned(y, ldy, size, rows) &&
                   rows_aligned(residual, ld_residual, ssize, rows) && rows_aligned(h, ldh, ssize, rows);
  // Up to 1,024 columns two units a warp and 24 warps on an SM; wider, where the warps of a row wait for one another, four units and
  // sixteen warps.  32,768 rows of 1,024 bfloat16 columns: 61.7 us, 70.4 us with four units; 8,192 rows of 4,096: 55.9 us, 73.7 us
  // with two units.  Beside a binary32 stream too: sixteen warps, which leave room for four rows of a team under way, take 65 to 66 us for
  // 32,768 rows of 520, 640 and 768 columns against 58 to 59 us, 15.5 us for 4,096 of 1,024 against 14.1 us, and for 32,768 of 1,000 and
  // of 1,024, the only sizes where they are faster, 70 to 78 us from run to run against 70 to 77 us, 3 % less on average.
  const Plan p = plan_of(cols, rows, {size, residual ? ssize : 0, 0}, cols <= 1024 || size + ssize == 8 ? 2 : 4,
                         cols <= 1024 ? 3 : 2, 2, 0, sms);
  a.ring = p.ring;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
#define REGTOPK_NORM(T, S, V, U) launch_norm<T, S, V, U>(a, p, dev, sms, s)
  return REGTOPK_BY_TYPE(REGTOPK_NORM);
#undef REGTOPK_NORM
}

// A slot for each block and group.
size_t regtopk_layer_norm_backward_workspace_bytes(int64_t rows, int64_t cols, int32_t groups) {
  if (rows < 0 || cols < 1 || cols > REGTOPK_NORM_MAX_COLS || groups < 1) return 0;
  return ((rows < kMostBackBlocks ? rows : kMostBackBlocks) + (size_t)groups) * 2 * cols * sizeof(float);
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
      (!offsets && groups != 1) || (uintptr_t)offsets % 8 || !make_drop(drop, &a.drop)) return REGTOPK_ERR_INVALID_ARG;
  if (cols > REGTOPK_NORM_MAX_COLS || groups > REGTOPK_NORM_MAX_GROUPS) return REGTOPK_ERR_TOO_LARGE;
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
  if (sms > kMostSms) sms = kMostSms;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  a.block_rows = 1;
  if (rows > 0) {
    a.source[0] = {static_cast<const char*>(dy), ld_dy * (int64_t)size};
    a.source[1] = {static_cast<const char*>(h), ldh * (int64_t)ssize};
    a.source[2] = {static_cast<const char*>(dh), ld_dh * (int64_t)ssize};
    a.mean = mean; a.rstd = rstd; a.weight = weight; a.dx = dx; a.dres = dresidual; a.ld_dx = ld_dx; a.ld_dres = ld_dresidual;
    a.rows = rows; a.cols = (int)cols; a.wide = (uintptr_t)weight % 16 == 0; a.groups = groups; a.offsets = offsets; a.partial = sums ? static_cast<float*>(workspace) : nullptr;
    const Plan p = plan_of(cols, rows, {size, ssize, dh ? ssize : 0}, size + ssize == 4 ? 4 : 2, 2, 1, 2, sms);
    a.ring = p.ring;
    const int64_t blocks = (int64_t)sms * (p.blocks < 4 ? p.blocks : 4), turns = (rows + blocks * p.ring.teams - 1) / (blocks * p.ring.teams);
    a.block_rows = turns * p.ring.teams;
    const bool vec = cols % 8 == 0 && rows_aligned(dy, ld_dy, size, rows) && rows_aligned(h, ldh, ssize, rows) &&
                     rows_aligned(dh, ld_dh, ssize, rows) && rows_aligned(dx, ld_dx, size, rows) &&
                     rows_aligned(dresidual, ld_dresidual, ssize, rows);
#define REGTOPK_NORM_BACK(T, S, V, U) launch_norm_back<T, S, V, U>(a, p, dev, s)
    const int rc = REGTOPK_BY_TYPE(REGTOPK_NORM_BACK);
#undef REGTOPK_NORM_BACK
    if (rc != REGTOPK_OK) return rc;
  }
  if (sums) {
    NormSumArgs n;
    n.partial = static_cast<const float*>(workspace); n.dweight = dweight; n.dbias = dbias; n.ld_dweight = ld_dweight; n.ld_dbias = ld_dbias;
    n.rows = rows; n.block_rows = a.block_rows; n.cols = (int)cols; n.accumulate = accumulate; n.offsets = offsets;
    return start(k_norm_sum, dim3((unsigned)((cols + 31) / 32), (unsigned)groups), dim3(32, kRuns), 0, s, n);
  }
  return REGTOPK_OK;
}

}  // extern "C"
