// Dropout and layer norm with their gradients (include/regtopk_train.h).
//
// All of them have memory traffic for their floor: a few operations per element and one read and one write of each array.
// So each kernel reads every input once, keeps many copies under way, and draws the dropout mask again wherever it is
// needed instead of storing it (one Philox call for eight columns costs less issue time than a byte of mask costs
// bandwidth).  Dropout reaches that floor.  The norms spend 40 to 46 instructions of a lane on a value at 16 to 24 warps an SM:
// little over half of the issue slots and of the memory's bandwidth are in use, and it is the latency between the two, with too few
// warps to hide it, that binds them.

#include "train_common.cuh"

namespace {

// ---- eight columns of a row ------------------------------------------------------------------------------------------
// This lane's columns of the unit that begins at column c0; past the end of the row zeros if VEC, `past` if not.  SHARED: the row is
// in shared memory, otherwise in global.
template <typename T, bool VEC, bool SHARED, typename Column>
__device__ __forceinline__ void read_eight(Octet& f, const T* row, Column c0, int lane, Column cols, float past = 0.0f) {
  if (VEC) {
    Eight<T> v;
    if (c0 + lane * 8 >= cols) v.clear();
    else if (SHARED) v.load(row + c0 + lane * 8);
    else v.fetch(row + c0 + lane * 8);
    v.get(f);
  } else {
    float e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = c0 + lane_col<false>(lane, j) < cols ? to_float(row[c0 + lane_col<false>(lane, j)]) : past;
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(e[2 * i], e[2 * i + 1]);
  }
}
template <typename T, bool VEC, typename Column>
__device__ __forceinline__ void store_eight(const Octet& f, T* row, Column c0, int lane, Column cols) {
  if (VEC) {
    Eight<T> v;
    v.put(f);
    if (c0 + lane * 8 < cols) v.store(row + c0 + lane * 8);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c0 + lane_col<false>(lane, j) < cols) row[c0 + lane_col<false>(lane, j)] = from_float<T>((j & 1) ? f[j >> 1].y : f[j >> 1].x);
  }
}

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

// ---- rows through shared memory ------------------------------------------------------------------------------------
// A team of warps takes one row at a time, U units of 256 columns a warp and eight columns a lane and unit.  The rows of
// up to three arrays come through a ring in shared memory by bulk asynchronous copies that the team's first lane issues
// `stages` rows ahead: what is under way then depends neither on registers nor on how long a row takes.  (Held in
// registers instead, 32,768 rows of 1,024 columns took 135 us in the backward pass with a warp per row, whose 216 registers
// leave room for eight warps on an SM, and 113 us with four warps per row and a barrier for every two rows.)
// A copy takes whole 16-byte words, those at both ends of an unaligned row included: the other bytes in them belong to
// the same allocation and are not looked at.
constexpr int kMostWarps = 16;   // of a block
constexpr int kMostStages = 4;

struct Source {  // one array's rows
  const char* p;
  int64_t pitch;  // bytes from row to row
};

struct RingShape {
  int warps, teams, stages;  // warps of a team, teams of a block, rows of a team under way
  int row_bytes[3];          // of each array, 0: not there
  int room[3];               // what a row of it takes in a stage
  int stage_bytes;
};

struct Team {
  int warps, index, warp, lane;  // its warps; this thread's team, warp within the team, lane
  int col0;                      // this warp's first column
  __device__ __forceinline__ Team(int warps_, int units) : warps(warps_) {
    const int w = threadIdx.x >> 5;
    index = w / warps;
    warp = w - index * warps;
    lane = threadIdx.x & 31;
    col0 = warp * units * 256;
  }
  __device__ __forceinline__ bool leads() const { return warp == 0 && lane == 0; }
  __device__ __forceinline__ void sync() const {
    if (warps == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(index + 1), "r"(warps * 32) : "memory");
  }
};

// Waits for a row that has not come yet.  If it does not, the team's first lane (`drains`) waits once more for all that is under
// way, because the shared memory is another block's after this one's end.  Stages without a copy come last and cost one more such
// wait in all.
__device__ __noinline__ bool ring_wait(u32 bars, u32 stage, u32 phase, int stages, volatile u32* quit, bool drains) {
  if (bar_wait_long(bars + stage * 8, phase, quit)) return true;
  for (int i = 0; i < stages && drains; ++i) {
    bar_wait(bars + stage * 8, phase, quit + 1);
    if (++stage == (u32)stages) {
      stage = 0;
      phase ^= 1;
    }
  }
  return false;
}

// A team's ring: it holds the rows first, first + step, ... below `end` of the arrays, one after the other.
// WALKS: where the copies go on from is kept in registers and goes from row to row by additions; otherwise it is worked out
// from the row.  The forward pass is faster with the former for most sizes (16,384 rows of 1,023 bfloat16 columns 48.0 us against
// 50.5 us, 20,000 of 232 float16 columns beside a binary32 stream 14.8 us against 15.7 us, but 6,000 of 1,000 bfloat16 columns 17.1 us
// against 15.7 us), the backward pass, which has no registers to spare, with the latter (2,048 rows of 8,192: 78 us against 83 us;
// 16,384 of 1,023: 70 us against 84 us).
template <bool WALKS> struct Ring {
  const RingShape& shape;
  const Source* source;
  char* base;
  u32 bars;
  volatile u32* quit;  // and in the word behind it: given up a second time
  int64_t step, end;
  u32 stage, phase;      // where the next row to be read lies
  const char* ahead[3];  // WALKS: of each array the row to be requested next,
  int64_t leap[3], left; //   bytes from one to the one after, and how many are left
  u32 low[3];            //   the low part of the address of the next row to be read

  __device__ __forceinline__ void request(int64_t row, u32 into) {  // the team's first lane only
    if (WALKS ? left <= 0 : row >= end) return;
    if (WALKS) --left;
    const u32 bar = bars + into * 8;
    u32 at = smem_at(base) + into * shape.stage_bytes, total = 0;
    u32 to[3], size[3];
    const char* from[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      size[i] = 0;
      if (!shape.row_bytes[i]) continue;
      const char* p = WALKS ? ahead[i] : source[i].p + row * source[i].pitch;
      const u32 skip = (u32)(uintptr_t)p & 15u;
      from[i] = p - skip;
      to[i] = at;
      size[i] = (skip + shape.row_bytes[i] + 15u) & ~15u;
      total += size[i];
      at += shape.room[i];
      if (WALKS) ahead[i] += leap[i];
    }
    bar_expect(bar, total);
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (size[i])
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                     ::"r"(to[i]), "l"(from[i]), "r"(size[i]), "r"(bar) : "memory");
  }
  // Waits for the next row.  Should it not come (see bar_wait), nothing more is requested, and the kernel runs to its end with what
  // there is.
  __device__ __forceinline__ void await(bool leads) {
    if (!bar_done(bars + stage * 8, phase) && !ring_wait(bars, stage, phase, shape.stages, quit, leads && (WALKS ? left : end) >= 0))
      (WALKS ? left : end) = -1;
  }
  // Array number `array` of the next row, which is row `row` of the arrays.
  template <typename T, bool VEC, bool RING> __device__ __forceinline__ const T* row_of(int64_t row, int array) const {
    if (!RING) return reinterpret_cast<const T*>(source[array].p + row * source[array].pitch);
    const char* p = base + stage * shape.stage_bytes;
    for (int i = 0; i < array; ++i) p += shape.room[i];
    if (!VEC) p += (WALKS ? low[array] : (u32)(uintptr_t)source[array].p + (u32)row * (u32)source[array].pitch) & 15u;
    return reinterpret_cast<const T*>(p);
  }
  // The next row, `row`, has been read by the whole team: its place is for the row `stages` rows on.
  __device__ __forceinline__ void pass(int64_t row, bool leads) {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (WALKS) low[i] += (u32)leap[i];
    if (leads) request(WALKS ? 0 : row + shape.stages * step, stage);
    if (++stage == (u32)shape.stages) {
      stage = 0;
      phase ^= 1;
    }
  }
};

// The weight vectors in shared memory, brought by 4-byte asynchronous copies (a view into a flat parameter vector is
// aligned no better) while the first rows are on their way.  VEC lanes read their eight columns as two 16-byte words;
// each half of a unit is stored contiguously over the lanes so that these reads meet no bank twice.
template <bool VEC> __device__ __forceinline__ int vector_place(int c) {
  return VEC ? (c & ~255) + ((c >> 2) & 1) * 128 + ((c >> 3) & 31) * 4 + (c & 3) : c;
}
template <bool VEC> __device__ __forceinline__ void fetch_vector(float* to, const float* from, int cols) {
  for (int c = threadIdx.x; c < (cols + 255 & ~255); c += blockDim.x) {  // zeros up to a whole unit
    float* dst = to + vector_place<VEC>(c);
    if (from && c < cols) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_at(dst)), "l"(from + c) : "memory");
    else *dst = 0.0f;
  }
}
template <bool VEC> __device__ __forceinline__ void read_vector(Octet& f, const float* from, int c0, int lane) {
  if (VEC) {
    const float4 lo = *reinterpret_cast<const float4*>(from + c0 + lane * 4);
    const float4 hi = *reinterpret_cast<const float4*>(from + c0 + 128 + lane * 4);
    f[0] = make_float2(lo.x, lo.y); f[1] = make_float2(lo.z, lo.w);
    f[2] = make_float2(hi.x, hi.y); f[3] = make_float2(hi.z, hi.w);
  } else {
    const float* p = from + c0 + lane;
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(p[64 * i], p[64 * i + 32]);
  }
}
// The same eight columns straight from global memory, for a team that has few rows.  `wide`: the vector is 16-byte aligned.  NULL:
// zeros.
template <bool VEC> __device__ __forceinline__ void load_vector(Octet& f, const float* from, bool wide, int c0, int lane, int cols) {
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = both(0.0f);
  if (!from) return;
  if (VEC && wide) {
    if (c0 + lane * 8 >= cols) return;
    const float4* p = reinterpret_cast<const float4*>(from + c0 + lane * 8);
    const float4 lo = p[0], hi = p[1];
    f[0] = make_float2(lo.x, lo.y); f[1] = make_float2(lo.z, lo.w);
    f[2] = make_float2(hi.x, hi.y); f[3] = make_float2(hi.z, hi.w);
  } else {
    float e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = c0 + lane_col<VEC>(lane, j) < cols ? from[c0 + lane_col<VEC>(lane, j)] : 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(e[2 * i], e[2 * i + 1]);
  }
}

// Shared memory of a block: barriers, values that the warps of a team exchange, vectors, rings.
struct Common {
  uint64_t bars[kMostWarps][kMostStages];  // [team][stage]
  float2 exchange[2][kMostWarps];          // two sets used in turn
  u32 quit[2];
};

__device__ __forceinline__ int padded(int cols) { return (cols + 255) & ~255; }

// Sets a team's ring up and requests its first rows.
template <bool RING, bool WALKS>
__device__ __forceinline__ Ring<WALKS> make_ring(Common& common, const RingShape& shape, const Source* source, char* rings, const Team& t,
                                                 int64_t first, int64_t step, int64_t end) {
  Ring<WALKS> ring{shape, source, rings + t.index * shape.stages * shape.stage_bytes, smem_at(&common.bars[t.index][0]), common.quit,
                   step, end, 0, 0};
  if (!RING) return ring;
  if (WALKS) {
    ring.left = first < end ? (end - first + step - 1) / step : 0;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      ring.ahead[i] = source[i].p + first * source[i].pitch;
      ring.leap[i] = step * source[i].pitch;
      ring.low[i] = (u32)(uintptr_t)ring.ahead[i];
    }
  }
  if (threadIdx.x == 0) common.quit[0] = common.quit[1] = 0;
  if (t.leads()) {
    for (int i = 0; i < shape.stages; ++i) bar_init(ring.bars + i * 8, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    for (int i = 0; i < shape.stages; ++i) ring.request(first + i * step, i);
  }
  return ring;
}

// a / b to binary32's accuracy by the reciprocal of b and one correction (Newton); exact where the quotient is a whole number.
__device__ __forceinline__ float quotient(float a, float b, float reciprocal) {
  const float q = a * reciprocal, better = fmaf(fmaf(-q, b, a), reciprocal, q);
  return better == better ? better : q;  // infinity
}
// 1 / sqrt(x) by the approximation and one step of Newton's method; where that has no value (0, infinity), the approximation.
// x is not halved: half of the smallest number is 0.
__device__ __forceinline__ float inverse_root(float x) {
  const float y = rsqrtf(x), better = fmaf(0.5f * y, fmaf(-x * y, y, 1.0f), y);
  return better == better ? better : y;
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
// How a row is shared and how the shared memory of an SM is divided.
//   rings: `blocks` blocks of eight warps on an SM (one of sixteen for the widest rows); a warp takes up to
//   `most_units` units.  `vectors` float32 vectors of the columns lie beside the rings, `joint` more where a block has two
//   teams or more.  Two rows of a team are under way, up to four where an SM has fewer than twelve teams (gradient of 4,096 rows of
//   4,096 binary32 columns, two teams to an SM: 76 us against 101 us; wide 16-bit rows lose 3 %, 2,000 of 8,192 take 42.5 us
//   against 41.2 us; with twelve teams, 6,000 rows of 1,000 bfloat16 columns only start later: 18.1 us against 17.1 us).
//   no rings, where no team of the rings would have a second row (or two rows do not fit): as many warps a row as it has units,
//   because then the time is nearly that of one row (backward pass, 1,000 rows of 1,000 columns: 14.3 us against 20.5 us with
//   four units a warp).  There are fewer teams then, so that one takes a few rows in turn: up to three of 1,024 bfloat16 columns, 592
//   teams where the rings have 1,776.  Rings from the second row on would take 5.9 us in place of 7.0 us for 1,500 such rows, and in the
//   backward pass 19.3 us in place of 16.6 us for 1,000 and 19.6 us in place of 18.0 us for 1,500.
struct Plan {
  int units, threads, blocks;
  size_t smem;
  bool rings;
  RingShape ring;
};
constexpr int kSmemOfSm = 227 * 1024, kSmemOfBlock = 2 * 1024;  // the latter: static, and what the system takes

inline Plan plan_of(int64_t cols, int64_t rows, const size_t (&size)[3], int most_units, int blocks, int vectors, int joint, int sms) {
  Plan p;
  const int n = (int)((cols + 255) / 256), column_bytes = n * 256 * (int)sizeof(float);
  p.ring.stage_bytes = 0;
  for (int i = 0; i < 3; ++i) {
    p.ring.row_bytes[i] = (int)(cols * size[i]);
    p.ring.room[i] = size[i] ? (p.ring.row_bytes[i] + 15 + 15) / 16 * 16 : 0;
    p.ring.stage_bytes += p.ring.room[i];
  }
  const auto share = [&](int units) {
    p.ring.warps = (n + units - 1) / units;
    p.units = (n + p.ring.warps - 1) / p.ring.warps;
  };
  share(n > most_units * kMostWarps ? 4 : most_units);
  const int warps = kMostWarps / 2;  // of a block
  p.blocks = p.ring.warps > warps ? 1 : blocks;
  int teams = p.ring.warps > warps ? 1 : warps / p.ring.warps;
  p.rings = rows > (int64_t)sms * p.blocks * teams;
  if (p.rings) {
    for (;; --teams) {
      p.smem = (size_t)column_bytes * (vectors + (teams > 1 ? joint : 0));
      const int stages = (kSmemOfSm / p.blocks - kSmemOfBlock - (int)p.smem) / (teams * p.ring.stage_bytes);
      const int most_stages = p.blocks * teams >= 12 ? 2 : kMostStages;
      p.ring.teams = teams;
      p.ring.stages = stages > most_stages ? most_stages : stages;
      if (stages >= 2) break;
      if (teams == 1) {
        if (p.blocks == 1) break;
        p.blocks = 1;  // a block alone on its SM
        teams = 2;
      }
    }
    p.smem += (size_t)p.ring.teams * p.ring.stages * p.ring.stage_bytes;
    p.rings = p.ring.stages >= 2;
  }
  if (!p.rings) {
    share(n <= kMostWarps ? 1 : n <= 2 * kMostWarps ? 2 : 4);
    const int64_t most = p.ring.warps >= 4 ? 1 : 4 / p.ring.warps, each = (rows + sms - 1) / sms;
    p.ring.teams = (int)(each < most ? each : most);
    p.ring.stages = 0;
    p.blocks = kMostWarps / (p.ring.warps * p.ring.teams);
    p.smem = (size_t)column_bytes * (vectors + (p.ring.teams > 1 ? joint : 0));
  }
  p.threads = 32 * p.ring.warps * p.ring.teams;
  return p;
}

template <auto kKernel> bool allow_smem(int dev) {
  static uint64_t done;  // of this kernel, one bit a device
  if (__atomic_load_n(&done, __ATOMIC_RELAXED) >> dev & 1) return true;
  if (cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemOfSm - kSmemOfBlock) != cudaSuccess) return false;
  __atomic_fetch_or(&done, 1ull << dev, __ATOMIC_RELAXED);
  return true;
}

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

// For the workspace's size, which is asked for without a device.
constexpr int kMostSms = 160, kMostBackBlocks = kMostSms * 4;

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
