// What the norms share: eight columns of a row, rows through rings in shared memory, groups of rows, the shape of a launch.
#ifndef REGTOPK_NORM_ROWS_CUH_
#define REGTOPK_NORM_ROWS_CUH_

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

// ---- groups of rows -------------------------------------------------------------------------------------------------
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

// For the workspace's size, which is asked for without a device.
constexpr int kMostSms = 160, kMostBackBlocks = kMostSms * 4;

}  // namespace
#endif
