// Products of tokens with the matrices of their experts, ragged groups, and the gradients to the matrices
// (include/regtopk_train.h), on the fifth-generation tensor cores.
//
// Both kernels are persistent, one block per SM or one pair of blocks for two: a warp that issues TMA copies, a warp that
// issues tcgen05.mma on the tiles that have landed, and warps that write finished accumulators while the next tile is
// multiplied.
//
//   k_rows     D[128 or 256 output features][up to 256 tokens] = W[features][k] X[tokens][k]^T.  The features take the
//              lanes of the accumulator; the tokens of a group, of which there may be any number, take its columns, whose
//              count the instruction chooses in steps of 16 (of 32 for a pair).  A lane then holds one feature, so that a
//              warp writes consecutive elements of a token's row.
//   k_weights  D[128 or 256 columns of x][up to 256 columns of dy] = sum over tokens; a lane holds one column of x, so
//              that a warp writes (or adds to) consecutive elements of a row of the gradient at any alignment.
//
// A pair divides the features (the columns of x) and the tokens (the columns of dy) of its tile: each block holds half of
// both operands, and the products of the first block read both halves.  Tiles lie in shared memory in the 128-byte
// swizzle, copied in boxes that are 64 elements (128 bytes) wide.
//
// What bounds them (B200, 1.3-1.9 GHz under its power limit): 32,768 tokens in 64 groups, 2,048 -> 2,304, 240 us or 1,290 TFLOP/s, 288 us
// or 1,070 where the power limit has set in; the tensor core is active for 77 % of the cycles.  The same loops without any copies take
// 219 us and a library's product of one dense group of the same sizes 209 us: groups that are no multiple of 256 tokens cost 5 %,
// tiles of 207 tokens on average the rest.

#include <cuda.h>
#include <string.h>

#include <type_traits>
#include <utility>

#include "train_common.cuh"

namespace {

// ---- PTX -------------------------------------------------------------------------------------------------------------
// Copies of boxes.  kCtas 2: the barrier may be the other block's of a pair.
template <int kCtas> __device__ __forceinline__ void tma_2d(u32 to, const CUtensorMap* map, u32 bar, int x, int y) {
  if constexpr (kCtas == 2)
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(to), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(to), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
template <int kCtas> __device__ __forceinline__ void tma_3d(u32 to, const CUtensorMap* map, u32 bar, int x, int y, int z) {
  if constexpr (kCtas == 2)
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(to), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(to), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
template <int kCtas> __device__ __forceinline__ void mma(u32 d, uint64_t a, uint64_t b, u32 how, bool add) {
  if constexpr (kCtas == 2)
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(how), "r"((u32)add) : "memory");
  else
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(how), "r"((u32)add) : "memory");
}
// Arrives on the barrier (of both blocks of a pair) when the products issued so far are done.
template <int kCtas> __device__ __forceinline__ void mma_commit(u32 bar) {
  if constexpr (kCtas == 2)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// The place in the first block of a pair that corresponds to one here.
template <int kCtas> __device__ __forceinline__ u32 in_first(u32 at) {
  if constexpr (kCtas == 1) return at;
  u32 there;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(there) : "r"(at));
  return there;
}
// Arrives on a barrier of the first block.  kOrders: what this thread has written is seen by who waits there.  Where that is
// nothing, because an accumulator has only been read, ordering would wait for all of this thread's stores to memory.
template <int kCtas, bool kOrders> __device__ __forceinline__ void bar_arrive_first(u32 bar) {
  if constexpr (kCtas == 1 && kOrders) bar_arrive(bar);
  else if constexpr (kCtas == 1) asm volatile("mbarrier.arrive.relaxed.cta.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
  else if constexpr (kOrders) asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(in_first<2>(bar)) : "memory");
  else asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(in_first<2>(bar)) : "memory");
}
template <int kCtas> __device__ __forceinline__ u32 cta_rank() {
  if constexpr (kCtas == 1) return 0;
  u32 r;
  asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
  return r;
}
// All threads of the block, or of both blocks of a pair.
template <int kCtas> __device__ __forceinline__ void sync_all() {
  if constexpr (kCtas == 1) __syncthreads();
  else asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 accumulator columns of this warp's 32 lanes.
__device__ __forceinline__ void tmem_read(float (&v)[32], u32 at) {
  u32 r[32];
  __syncwarp();
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at) : "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// 16 of them.
__device__ __forceinline__ void tmem_read16(float (&v)[16], u32 at) {
  u32 r[16];
  __syncwarp();
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(at) : "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// ---- descriptors -----------------------------------------------------------------------------------------------------
// Shared memory operand in the 128-byte swizzle: start, distance of 64-element blocks along the operand's own rows
// (used where those are the contiguous dimension), distance of groups of eight swizzled lines, in bytes.
__device__ __forceinline__ uint64_t operand(u32 at, u32 leading, u32 stride) {
  const u32 lo = at >> 4 | leading >> 4 << 16, hi = stride >> 4 | 1u << 14 | 2u << 29;  // shared addresses are below 2^18
  return (uint64_t)hi << 32 | lo;
}
// One lane of a converged warp.  The warp that issues products runs as a whole and elects a lane for the instructions
// themselves: its addresses and descriptors are then uniform, which the instructions want (with a single thread in the
// loop a stage of four products took 430 ns to issue, however few columns they had).
__device__ __forceinline__ bool elected() {
  u32 yes;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(yes));
  return yes;
}
constexpr int kBox = 64;                   // elements of a line of a box: 128 bytes
// Of the summed dimension in a stage.  Two lines of a box deep where that dimension is the contiguous one: a stage of 64
// holds too little work for what it costs to wait for it, issue it and hand it back.
constexpr int kDepth = 128;
constexpr int kBoxBytes = kBox * kDepth * 2;  // a box whose lines are the summed dimension
constexpr int kStepBytes = 16 * kBox * 2;     // from one step of sixteen such lines to the next
constexpr int kLanes = 128;                // accumulator lanes: the fixed side of a tile

// Instruction descriptor: binary32 accumulators, both operands of one 16-bit type, 128 lanes of each block, `columns`
// columns; _mn: the operand's own rows, not the summed dimension, are contiguous.
template <int kCtas> __device__ __forceinline__ u32 instruction(bool bf16, bool a_mn, bool b_mn, int columns) {
  return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (u32)a_mn << 15 | (u32)b_mn << 16 | (u32)(columns >> 3) << 17 | (u32)(kCtas * kLanes >> 4) << 24;
}

// The products of one stage, up to eight steps of sixteen of the summed dimension.  An operand whose own rows are contiguous
// (kMn) lies in boxes whose lines are the summed dimension; the other kind in two halves of 64 of it, `half` bytes apart.
template <bool kMn> __device__ __forceinline__ uint64_t step_of(uint64_t operand, int i, u32 half) {
  return operand + ((kMn ? i * kStepBytes : (i >> 2) * half + (i & 3) * 32) >> 4);
}
template <int kCtas, bool kMnA, bool kMnB>
__device__ __forceinline__ void multiply(u32 acc, uint64_t a, u32 half_a, uint64_t b, u32 half_b, u32 how, int steps, bool begins) {
  if (steps == kDepth / 16) {
#pragma unroll
    for (int i = 0; i < kDepth / 16; ++i) mma<kCtas>(acc, step_of<kMnA>(a, i, half_a), step_of<kMnB>(b, i, half_b), how, i || !begins);
  } else {
    for (int i = 0; i < steps; ++i) mma<kCtas>(acc, step_of<kMnA>(a, i, half_a), step_of<kMnB>(b, i, half_b), how, i || !begins);
  }
}

// Columns come in steps of sixteen, thirty-two for a pair.
template <int kCtas> __device__ __forceinline__ int rounded(int columns) { return (columns + 16 * kCtas - 1) / (16 * kCtas) * (16 * kCtas); }

// Warp 0 copies, warp 1 multiplies, warp 2 keeps the TMEM, warp 3 clears; the others write, some for each quarter of the
// lanes: two where the outputs are rounded to 16 bits (four are no faster), four for the weight gradients, where the time goes
// into waiting for loads and stores (32,768 tokens over 32 matrices of 1024 x 2304: 183 us against 221 us with two).
constexpr int kRowShare = 2, kWeightShare = 4;
constexpr int threads_of(int share) { return 128 + 128 * share; }

// `full`, `masked`, `free_` and `last` are the first block's of a pair alone; the other block's copies and warps arrive there too.
template <int kStages> struct Shared {
  uint64_t full[kStages], empty[kStages];   // a stage has landed; has been used
  uint64_t landed[kStages], masked[kStages]; // k_weights: this block's part of a group's last tokens has landed; all of it has been masked
  uint64_t done[2], free_[2], last;          // an accumulator is finished; has been read; all products are done
  u32 tmem, quit;
};

// No block takes TMEM before the kernel before it has ended, or lets a kernel behind it start before it has taken its own: whoever
// waits for the other then holds none that the other needs.
template <int kCtas, int kStages> __device__ __forceinline__ void set_up(Shared<kStages>& sh, int tmem_columns, int readers) {
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      bar_init(smem_at(&sh.full[i]), 1);
      bar_init(smem_at(&sh.empty[i]), 1);
      bar_init(smem_at(&sh.landed[i]), 1);
      bar_init(smem_at(&sh.masked[i]), kCtas);
    }
    for (int i = 0; i < 2; ++i) {
      bar_init(smem_at(&sh.done[i]), 1);
      bar_init(smem_at(&sh.free_[i]), readers * kCtas);
    }
    bar_init(smem_at(&sh.last), 1);
    sh.quit = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  await_predecessor();
  if (threadIdx.x >> 5 == 2) {
    if constexpr (kCtas == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&sh.tmem)), "r"(tmem_columns) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&sh.tmem)), "r"(tmem_columns) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
  }
  tmem_fence_before();
  __syncthreads();
  sync_all<kCtas>();
  tmem_fence_after();
  let_successor_start();
}
// No block of a pair leaves before the other: its barriers and its shared memory are in use until then.
template <int kCtas, int kStages> __device__ __forceinline__ void tear_down(Shared<kStages>& sh, int tmem_columns) {
  tmem_fence_before();
  __syncthreads();
  sync_all<kCtas>();
  tmem_fence_after();
  if (threadIdx.x >> 5 == 2) {
    if constexpr (kCtas == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(sh.tmem), "r"(tmem_columns));
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(sh.tmem), "r"(tmem_columns));
  }
}

// The copying thread at its end: `turn` stages have been filled.  It waits until each of them has been used, so that nothing is
// under way when the block ends; if the block has given up, until what was requested has landed.  In a pair the first
// block's barriers say so for both, and the second block waits for the first at the end.  Bits of `ended`: the stage
// was last filled with the end of a group (k_weights), whose landing `landed` tells; bits of `odd`: it did so an odd number of times.
template <int kStages> __device__ __forceinline__ void drain(Shared<kStages>& sh, u32 turn, bool first, u32 ended, u32 odd) {
  volatile u32* quit = &sh.quit;
  const u32 from = turn > (u32)kStages ? turn - kStages : 0;
  for (u32 t = from; t < turn; ++t) {
    u32 never = 0;
    const u32 s = t % kStages, parity = (t / kStages) & 1;
    if (!*quit && bar_wait(smem_at(&sh.empty[s]), parity, quit)) continue;
    if (ended >> s & 1) bar_wait(smem_at(&sh.landed[s]), (odd >> s & 1) ^ 1, &never);
    else if (first) bar_wait(smem_at(&sh.full[s]), parity, &never);
  }
}

// The multiplying thread, when the block has given up: no product may be under way when the block ends.
template <int kCtas, int kStages> __device__ __forceinline__ void settle(Shared<kStages>& sh) {
  u32 never = 0;
  mma_commit<kCtas>(smem_at(&sh.last));
  bar_wait(smem_at(&sh.last), 0, &never);
}

__device__ __forceinline__ int64_t limited(int64_t v, int64_t rows) { return v < 0 ? 0 : v > rows ? rows : v; }

// ---- y[t] = w x[t] -----------------------------------------------------------------------------------------------------
struct RowsArgs {
  const int64_t* offsets;
  void* y;
  int64_t ldy;
  int groups, weights, rows, k, m;
  int shared_weights;  // all matrices are the first one
  int pairs;           // two neighbouring elements of y may be written as one word
  // The summed dimension is divided into `parts` of `part_k`, each a tile of its own whose sums go to partial [parts][rows][m].
  int parts, part_k;
  float* partial;
};

// Terms that one accumulator of k_rows sums before the sum moves on to registers (kWeightsChain, below, says why).  Outputs are rounded
// to 16 bits, so that this may be more than for the weight gradients: 4,096 terms of one sign come out 2.6e-5 too small, a tenth of half
// a step of float16 and less of bfloat16; without a limit 65,536 terms came out 4e-4 too small, nearly half a step.  Up to here a kernel
// without those registers does it; longer sums take 0 to 4 % more time than they would in it (8,192 tokens over 16 matrices of 2304 x 8192: 312 us against
// 308 us; with 2,048 terms 1 % more, and sums of 2,144 over 91 groups of 16 tokens in all 13.5 us in place of 12.1 us).
constexpr int kRowsChain = 4096;
// Writing warps for each quarter of the lanes: twice as many share the sums in registers.
template <bool kLong> constexpr int kRowShareOf = kLong ? 2 * kRowShare : kRowShare;
template <bool kLong> constexpr int kRowThreadsOf = threads_of(kRowShareOf<kLong>);
constexpr int kTableGroups = REGTOPK_MATMUL_MAX_GROUPS;

// How a group's rows are cut: as many tiles as the widest allows, all of one size but the last.
__device__ __forceinline__ int tile_rows(int count, int most) {
  const int tiles = (count + most - 1) / most;
  return tiles ? (int)(((u32)count + (u32)tiles - 1) / (u32)tiles + 15) & ~15 : 16;  // count + tiles may pass 2^31
}

// The tiles of a pair (or a block), every `pairs`-th of all: for each tile of tokens those of the features one after the other.
// Each warp walks through them by additions.
struct RowWalk {
  int token_tiles, feature_tiles, step_tokens, step_features;
  int parts;                       // `in` counts parts of a tile of features
  int at, in, group;               // tile of tokens, tile of features; the former's group
  int row, count, feature;         // the tile: first token, tokens, first feature
  const int *before, *start, *end; // of each group in the table's order: tiles of tokens before it, its rows
  template <int kMost, int kCtas> __device__ __forceinline__ void find() {
    if (at >= token_tiles) return;
    while (at >= before[group + 1]) ++group;
    const int step = tile_rows(end[group] - start[group], kMost);
    row = start[group] + (at - before[group]) * step;
    count = min(step, end[group] - row);
    feature = in / parts * (kCtas * kLanes);
  }
  __device__ __forceinline__ int part() const { return in % parts; }
  template <int kMost, int kCtas> __device__ __forceinline__ void next() {
    at += step_tokens;
    in += step_features;
    if (in >= feature_tiles) {
      in -= feature_tiles;
      ++at;
    }
    find<kMost, kCtas>();
  }
};

// The tokens of a tile, of which there are up to kMost, are divided between the blocks of a pair.
template <int kMost, int kCtas> struct RowStage {
  static constexpr int kTokens = kMost / kCtas, kBytesA = kLanes * kDepth * 2, kBytes = kBytesA + kTokens * kDepth * 2;
  static constexpr int kHalfA = kBytesA / 2, kHalfB = kTokens * kBox * 2;
  static constexpr int kCount = kTokens == 128 ? 3 : kTokens == 64 ? 4 : 5;
  static constexpr int kSmem = kCount * kBytes + 1024;
};

// kLong: for sums of more than kRowsChain terms.
template <typename T, int kMost, bool kTransposed, int kCtas, bool kLong>
__global__ void __launch_bounds__(kRowThreadsOf<kLong>, 1) k_rows(const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map, const RowsArgs a) {
  typedef RowStage<kMost, kCtas> Stage;
  constexpr int kStages = Stage::kCount, kBytesA = Stage::kBytesA, kBytes = Stage::kBytes;
  constexpr int kBoxRows = Stage::kTokens < 64 ? Stage::kTokens : 64;  // tokens of one copy
  constexpr int kTmem = 2 * kMost, kShare = kRowShareOf<kLong>, kRowThreads = kRowThreadsOf<kLong>;
  constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
  extern __shared__ uint8_t raw[];
  __shared__ Shared<kStages> sh;
  __shared__ int before[kTableGroups + 1], start[kTableGroups], end[kTableGroups];
  __shared__ int scan[kRowThreads / 32];
  const u32 tiles_at = (smem_at(raw) + 1023) & ~1023u;
  const int warp = __shfl_sync(kAll, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

  const u32 rank = cta_rank<kCtas>();

  set_up<kCtas>(sh, kTmem, 4 * kShare);
  // where each group's rows lie and how many tiles come before it; groups that share a matrix one after the other, so that
  // it is read from memory once (four workers over sixteen matrices of 9 MB: 752 MB read without that, 285 MB are needed)
  constexpr int kPer = (kTableGroups + kRowThreads - 1) / kRowThreads;  // groups of a thread
  {
    int own[kPer], sum = 0;
    const int per = (a.groups + kRowThreads - 1) / kRowThreads, sharers = a.groups / a.weights;
    for (int i = 0; i < per; ++i) {
      const int g = threadIdx.x * per + i;
      own[i] = 0;
      if (g < a.groups) {
        const int of = (g % sharers) * a.weights + g / sharers;  // in the table the groups of one matrix are neighbours
        const int lo = (int)limited(a.offsets[of], a.rows);
        int hi = (int)limited(a.offsets[of + 1], a.rows);
        if (hi < lo) hi = lo;
        start[g] = lo;
        end[g] = hi;
        const int step = tile_rows(hi - lo, kMost);
        own[i] = (hi - lo + step - 1) / step;
        sum += own[i];
      }
    }
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(kAll, upto, o);
      if (lane >= o) upto += v;
    }
    if (lane == 31) scan[warp] = upto;
    __syncthreads();
    for (int w = 0; w < warp; ++w) upto += scan[w];
    upto -= sum;
    for (int i = 0; i < per; ++i) {
      const int g = threadIdx.x * per + i;
      if (g < a.groups) {
        before[g] = upto;
        upto += own[i];
        if (g == a.groups - 1) before[a.groups] = upto;
      }
    }
    __syncthreads();
  }
  const int feature_tiles = (a.m + kCtas * kLanes - 1) / (kCtas * kLanes) * a.parts;
  const int pair = blockIdx.x / kCtas, pairs = gridDim.x / kCtas, tiles = before[a.groups];
  RowWalk t{tiles, feature_tiles, pairs / feature_tiles, pairs % feature_tiles, a.parts, pair / feature_tiles, pair % feature_tiles, 0, 0, 0, 0, before, start, end};
  t.find<kMost, kCtas>();
  volatile u32* quit = &sh.quit;

  if (warp == 0) {
    u32 s = 0, parity = 1, turn = 0;
    bool ok = true;
    const u32 full = in_first<kCtas>(smem_at(&sh.full[0]));
    for (; t.at < tiles; t.next<kMost, kCtas>()) {
      const int e = a.shared_weights ? 0 : t.group / (a.groups / a.weights);
      const int here = rounded<kCtas>(t.count) / kCtas, boxes = (here + kBoxRows - 1) / kBoxRows;  // this block's tokens
      const int feature = t.feature + (int)rank * kLanes, row = t.row + (int)rank * here;
      const int k0 = t.part() * a.part_k, k1 = min(a.k, k0 + a.part_k);
      for (int d = k0; d < k1; d += kDepth) {
        ok = ok && bar_wait(smem_at(&sh.empty[s]), parity, quit);
        __syncwarp();
        if (elected() && ok) {
          const int halves = k1 - d > kBox ? 2 : 1;
          const u32 at = tiles_at + s * kBytes, bar = full + s * 8;
          if (rank == 0)
            bar_expect(smem_at(&sh.full[s]), kCtas * ((kTransposed ? 2 : halves) * Stage::kHalfA + halves * boxes * kBoxRows * kBox * 2));
          if (kTransposed) {
            tma_3d<kCtas>(at, &w_map, bar, feature, d, e);
            tma_3d<kCtas>(at + kBoxBytes, &w_map, bar, feature + kBox, d, e);
          }
          for (int h = 0; h < halves; ++h) {
            if (!kTransposed) tma_3d<kCtas>(at + h * Stage::kHalfA, &w_map, bar, d + h * kBox, feature, e);
            for (int i = 0; i < boxes; ++i)
              tma_2d<kCtas>(at + kBytesA + h * Stage::kHalfB + i * kBoxRows * kBox * 2, &x_map, bar, d + h * kBox, row + i * kBoxRows);
          }
        }
        __syncwarp();
        turn += ok;
        if (++s == kStages) {
          s = 0;
          parity ^= 1;
        }
      }
    }
    if (elected()) drain(sh, turn, rank == 0, 0, 0);
  } else if (warp == 1) {
    if (rank == 0) {
      u32 s = 0, parity = 0, n = 0;
      bool ok = true;
      const auto take_accumulator = [&] {
        ok = ok && bar_wait(smem_at(&sh.free_[n & 1]), ((n >> 1) & 1) ^ 1, quit);
        tmem_fence_after();
      };
      for (; t.at < tiles; t.next<kMost, kCtas>(), ++n) {
        const u32 how = instruction<kCtas>(kBf16, kTransposed, false, rounded<kCtas>(t.count));
        u32 acc = sh.tmem + (n & 1) * kMost;
        take_accumulator();
        const int k0 = t.part() * a.part_k, k1 = min(a.k, k0 + a.part_k);
        bool begins = true;
        for (int d = k0; d < k1; d += kDepth) {
          ok = ok && bar_wait(smem_at(&sh.full[s]), parity, quit);
          __syncwarp();
          const bool ends = d + kDepth >= k1, moves = kLong && !ends && (d - k0 + kDepth) % kRowsChain == 0;
          if (elected() && ok) {
            const u32 at = tiles_at + s * kBytes;
            multiply<kCtas, kTransposed, false>(acc, operand(at, kTransposed ? kBoxBytes : 0, 1024), Stage::kHalfA,
                                                operand(at + kBytesA, 0, 1024), Stage::kHalfB, how, (min(kDepth, k1 - d) + 15) >> 4, kLong ? begins : d == k0);
            mma_commit<kCtas>(smem_at(&sh.empty[s]));
            if (ends || moves) mma_commit<kCtas>(smem_at(&sh.done[n & 1]));
          }
          __syncwarp();
          begins = moves;
          if (moves) {  // on to the other accumulator
            ++n;
            acc = sh.tmem + (n & 1) * kMost;
            take_accumulator();
          }
          if (++s == kStages) {
            s = 0;
            parity ^= 1;
          }
        }
      }
      if (elected() && !ok) settle<kCtas>(sh);
    }
  } else if (warp == 3 && a.parts == 1) {  // rows of no group
    const int64_t head = a.groups ? limited(a.offsets[0], a.rows) : a.rows, tail = limited(a.offsets[a.groups], a.rows);
    T* y = static_cast<T*>(a.y);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
      if (row >= head && row < tail) {
        row += (tail - 1 - row) / gridDim.x * gridDim.x;  // on to the last one before the tail
        continue;
      }
      for (int c = lane; c < a.m; c += 32) y[row * a.ldy + c] = from_float<T>(0.0f);
    }
  } else if (warp >= 4) {
    u32 n = 0;
    const int part = warp & 3, first = ((warp >> 2) - 1) * 32;  // the lanes that this warp may read, and its first columns
    const u32 swap = (lane & 1) ? 0x3276 : 0x5410;
    T* y = static_cast<T*>(a.y);
    const auto write = [&](const float (&v)[32], int f, int c0) {
      T* to = y + (int64_t)(t.row + c0) * a.ldy + f;
      const int left = f < a.m ? t.count - c0 : 0;
      if (a.parts > 1) {
        float* sums = a.partial + ((int64_t)t.part() * a.rows + t.row + c0) * a.m + f;
#pragma unroll
        for (int c = 0; c < 32; ++c) {
          if (c < left) *sums = v[c];
          sums += a.m;
        }
      } else if (a.pairs) {  // lanes of a pair of features exchange halves of two tokens, and each writes one token's pair
        const int odd = lane & 1;
        to += odd * (a.ldy - 1);
#pragma unroll
        for (int c = 0; c < 32; c += 2) {
          const u32 own = packed(v[c], v[c + 1], T()), other = __shfl_xor_sync(kAll, own, 1);
          if (c + odd < left) *reinterpret_cast<u32*>(to) = __byte_perm(own, other, swap);
          to += 2 * a.ldy;
        }
      } else {
#pragma unroll
        for (int c = 0; c < 32; ++c) {
          if (c < left) *to = from_float<T>(v[c]);
          to += a.ldy;
        }
      }
    };
    const auto await_sum = [&] {
      bar_wait(smem_at(&sh.done[n & 1]), (n >> 1) & 1, quit);  // given up: go on with what there is
      __syncwarp();
      tmem_fence_after();
    };
    const auto pass_sum = [&] {
      tmem_fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive_first<kCtas, false>(smem_at(&sh.free_[n & 1]));
    };
    for (; t.at < tiles; t.next<kMost, kCtas>()) {
      const int f = t.feature + (int)rank * kLanes + part * 32 + lane;
      if constexpr (kLong) {
        constexpr int kChunks = (kMost + 32 * kShare - 1) / (32 * kShare);
        float sum[kChunks][32];
#pragma unroll
        for (int i = 0; i < kChunks; ++i)
#pragma unroll
          for (int c = 0; c < 32; ++c) sum[i][c] = 0.0f;
        const int summed = min(a.part_k, a.k - t.part() * a.part_k);
        for (int d = 0; d < summed; d += kRowsChain, ++n) {
          await_sum();
#pragma unroll
          for (int i = 0; i < kChunks; ++i)
#pragma unroll
            for (int c0 = 0; c0 < 32; c0 += 16) {
              const int at = first + i * 32 * kShare + c0;
              if (at >= t.count) continue;
              float v[16];
              tmem_read16(v, sh.tmem + (n & 1) * kMost + at + ((u32)(part * 32) << 16));
#pragma unroll
              for (int c = 0; c < 16; ++c) sum[i][c0 + c] += v[c];
            }
          pass_sum();
        }
#pragma unroll
        for (int i = 0; i < kChunks; ++i)
          if (first + i * 32 * kShare < t.count) write(sum[i], f, first + i * 32 * kShare);
      } else {
        await_sum();
        for (int c0 = first; c0 < t.count; c0 += 32 * kShare) {
          float v[32];
          tmem_read(v, sh.tmem + (n & 1) * kMost + c0 + ((u32)(part * 32) << 16));
          write(v, f, c0);
        }
        pass_sum();
        ++n;
      }
    }
  }
  tear_down<kCtas>(sh, kTmem);
}

// ---- out[g] (+)= sum of dy[t] x[t]^T -------------------------------------------------------------------------------------
struct WeightsArgs {
  const int64_t* offsets;
  float* out;
  int64_t ld_out, inner_stride, outer_stride;
  int groups, inner, rows, k, m, accumulate;
  // The rows of a group are divided into `parts`, each a tile of its own, whose matrices lie part_stride apart.
  int parts;
  int64_t part_stride;
};

// Tokens that one accumulator sums.  The tensor core cuts the running sum off at every step of sixteen products
// instead of rounding it, so its error grows with the number of steps and always to the same side: 1.8e-5 of the result
// after 6,000 tokens of one sign.  After this many tokens the sum moves on to registers, where additions round: 2.4e-7 for
// values of one sign, 4.8e-7 for normal ones (256 tokens: 8e-8 and 2.4e-7, but 164 us where this takes 147 us, for 4,096
// tokens in each of eight groups; 1,024: 1e-6).
constexpr int kWeightsChain = 512;
constexpr int kWeightThreads = threads_of(kWeightShare);
constexpr int kWeightsMost = 256;
template <int kCtas> struct WeightStage {  // the columns of dy are divided between the blocks of a pair
  static constexpr int kBytesA = kLanes * kDepth * 2, kBytes = kBytesA + kWeightsMost / kCtas * kDepth * 2;
  static constexpr int kCount = kCtas == 2 ? 3 : 2;
  static constexpr int kSmem = kCount * kBytes + 1024;
};

// The tiles of a pair (or a block), every `pairs`-th of all: for each group the tiles of its matrix.
struct WeightWalk {
  int groups, k_tiles, tiles, step_groups, step_tiles;  // tiles: of a matrix, times `parts`
  int group, in;
  int row, count, k, m, columns;  // the tile: its group's rows; first column of x, first column and columns of dy
  const int2* rows;               // of each group: first row, number of rows
  int all_m, parts;
  __device__ __forceinline__ int part() const { return in % parts; }
  template <int kCtas> __device__ __forceinline__ void find() {
    if (group >= groups) return;
    row = rows[group].x;
    count = rows[group].y;
    if (parts > 1) {  // whole stages but for the last part
      const int each = ((count + parts - 1) / parts + kDepth - 1) / kDepth * kDepth, before = min(count, part() * each);
      row += before;
      count = min(each, count - before);
    }
    const int tile = in / parts;
    m = tile / k_tiles * kWeightsMost;
    k = tile % k_tiles * (kCtas * kLanes);
    columns = min(kWeightsMost, all_m - m);
  }
  template <int kCtas> __device__ __forceinline__ void next() {
    group += step_groups;
    in += step_tiles;
    if (in >= tiles) {
      in -= tiles;
      ++group;
    }
    find<kCtas>();
  }
};

// 32,768 tokens in 32 groups, 1,024 x 2,304, into rows of eight workers: 193 to 199 us, 780 to 800 TFLOP/s; added to what the rows hold, 227 to 232 us.  The products wait for
// accumulators on their way through registers and for the gradient's 302 MB (tensor core active for 46 % of the cycles).
template <typename T, int kCtas>
__global__ void __launch_bounds__(kWeightThreads, 1) k_weights(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap dy_map, const WeightsArgs a) {
  typedef WeightStage<kCtas> Stage;
  constexpr int kStages = Stage::kCount, kMost = kWeightsMost, kTmem = 2 * kMost;
  constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
  extern __shared__ uint8_t raw[];
  __shared__ Shared<kStages> sh;
  __shared__ int2 rows[kTableGroups];
  const u32 tiles_at = (smem_at(raw) + 1023) & ~1023u;
  const int warp = __shfl_sync(kAll, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const u32 rank = cta_rank<kCtas>();
  set_up<kCtas>(sh, kTmem, 4 * kWeightShare);
  for (int g = threadIdx.x; g < a.groups; g += kWeightThreads) {
    const int lo = (int)limited(a.offsets[g], a.rows), hi = (int)limited(a.offsets[g + 1], a.rows);
    rows[g] = make_int2(lo, max(hi - lo, 0));
  }
  __syncthreads();
  const int k_tiles = (a.k + kCtas * kLanes - 1) / (kCtas * kLanes), m_tiles = (a.m + kMost - 1) / kMost, matrix = k_tiles * m_tiles * a.parts;
  const int pair = blockIdx.x / kCtas, pairs = gridDim.x / kCtas;
  WeightWalk t{a.groups, k_tiles, matrix, pairs / matrix, pairs % matrix, pair / matrix, pair % matrix, 0, 0, 0, 0, 0, rows, a.m, a.parts};
  t.find<kCtas>();
  volatile u32* quit = &sh.quit;

  if (warp == 0) {
    u32 s = 0, parity = 1, turn = 0, ended = 0, odd = 0;
    bool ok = true;
    const u32 full = in_first<kCtas>(smem_at(&sh.full[0]));
    for (; t.group < a.groups; t.next<kCtas>()) {
      const int half = rounded<kCtas>(t.columns) / kCtas, boxes = (half + kBox - 1) / kBox;  // this block's columns of dy
      const int k = t.k + (int)rank * kLanes, m = t.m + (int)rank * half;
      for (int d = 0; d < t.count; d += kDepth) {
        const bool end = t.count - d < kDepth && (t.count - d) % 16;
        ok = ok && bar_wait(smem_at(&sh.empty[s]), parity, quit);
        __syncwarp();
        if (elected() && ok) {
          // the end of a group is masked first, by a warp of the block that has it
          const u32 at = tiles_at + s * Stage::kBytes, bytes = Stage::kBytesA + boxes * kBoxBytes;
          const u32 bar = end ? smem_at(&sh.landed[s]) : full + s * 8;
          if (end) bar_expect(smem_at(&sh.landed[s]), bytes);
          if (rank == 0) bar_expect(smem_at(&sh.full[s]), end ? 0 : kCtas * bytes);
          tma_2d<kCtas>(at, &x_map, bar, k, t.row + d);
          tma_2d<kCtas>(at + kBoxBytes, &x_map, bar, k + kBox, t.row + d);
          for (int i = 0; i < boxes; ++i) tma_2d<kCtas>(at + Stage::kBytesA + i * kBoxBytes, &dy_map, bar, m + i * kBox, t.row + d);
        }
        __syncwarp();
        turn += ok;
        ended = (ended & ~(1u << s)) | (u32)end << s;
        odd ^= (u32)end << s;
        if (++s == kStages) {
          s = 0;
          parity ^= 1;
        }
      }
    }
    if (elected()) drain(sh, turn, rank == 0, ended, odd);
  } else if (warp == 1) {
    if (rank == 0) {
      u32 s = 0, parity = 0, n = 0, odd = 0;  // odd: a bit for each stage, whether an odd number of groups has ended in it
      bool ok = true;
      for (; t.group < a.groups; t.next<kCtas>()) {
        const u32 how = instruction<kCtas>(kBf16, true, true, rounded<kCtas>(t.columns));
        for (int d = 0; d < t.count; d += kDepth) {
          const bool begins = d % kWeightsChain == 0, ends = (d + kDepth) % kWeightsChain == 0 || d + kDepth >= t.count;
          const int here = min(kDepth, t.count - d);
          if (begins) {
            ok = ok && bar_wait(smem_at(&sh.free_[n & 1]), ((n >> 1) & 1) ^ 1, quit);
            tmem_fence_after();
          }
          ok = ok && bar_wait(smem_at(&sh.full[s]), parity, quit);
          if (here & 15) {
            ok = ok && bar_wait(smem_at(&sh.masked[s]), (odd >> s) & 1, quit);
            if (kCtas == 2) asm volatile("fence.acq_rel.cluster;" ::: "memory");
            odd ^= 1u << s;
          }
          __syncwarp();
          if (elected() && ok) {
            const u32 at = tiles_at + s * Stage::kBytes;
            multiply<kCtas, true, true>(sh.tmem + (n & 1) * kMost, operand(at, kBoxBytes, 1024), 0,
                                        operand(at + Stage::kBytesA, kBoxBytes, 1024), 0, how, (here + 15) >> 4, begins);
            mma_commit<kCtas>(smem_at(&sh.empty[s]));
            if (ends) mma_commit<kCtas>(smem_at(&sh.done[n & 1]));
          }
          __syncwarp();
          if (ends) ++n;
          if (++s == kStages) {
            s = 0;
            parity ^= 1;
          }
        }
      }
      if (elected() && !ok) settle<kCtas>(sh);
    }
  } else if (warp == 3) {
    // The last lines of a group's last copy belong to the next group, whose values may be anything: zeros in their place, up
    // to the sixteen lines that a product takes.
    u32 s = 0, odd = 0;
    bool ok = true;
    for (; t.group < a.groups; t.next<kCtas>()) {
      if (!t.count) continue;
      s = (s + (t.count - 1) / kDepth) % kStages;  // the stage of its last copy
      if (t.count & 15) {
        const u32 at = tiles_at + s * Stage::kBytes + (t.count % kDepth) * 128;
        const int lines = 16 - (t.count & 15), boxes = 2 + (rounded<kCtas>(t.columns) / kCtas + kBox - 1) / kBox;
        ok = ok && bar_wait(smem_at(&sh.landed[s]), (odd >> s) & 1, quit);
        for (int box = 0; box < boxes && ok; ++box)
          for (int i = lane; i < lines * 8; i += 32)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + box * kBoxBytes + i * 16), "r"(0) : "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (elected() && ok) bar_arrive_first<kCtas, true>(smem_at(&sh.masked[s]));
        odd ^= 1u << s;
      }
      if (++s == kStages) s = 0;
    }
  } else if (warp >= 4) {
    u32 n = 0;
    constexpr int kOwn = kMost / kWeightShare;
    const int part = warp & 3, c0 = ((warp >> 2) - 1) * kOwn;  // this warp's lanes, and the first of its columns
    const u32 from = sh.tmem + c0 + ((u32)(part * 32) << 16);
    for (; t.group < a.groups; t.next<kCtas>()) {
      const int k = t.k + (int)rank * kLanes + part * 32 + lane, columns = t.columns - c0;  // may be none
      float sum[kOwn];
#pragma unroll
      for (int c = 0; c < kOwn; ++c) sum[c] = 0.0f;
      for (int d = 0; d < t.count; d += kWeightsChain, ++n) {
        bar_wait(smem_at(&sh.done[n & 1]), (n >> 1) & 1, quit);  // given up: go on with what there is
        __syncwarp();
        tmem_fence_after();
#pragma unroll
        for (int c = 0; c < kOwn; c += 16) {
          if (c < columns) {
            float v[16];
            tmem_read16(v, from + (n & 1) * kMost + c);
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[c + i] += v[i];
          }
        }
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive_first<kCtas, false>(smem_at(&sh.free_[n & 1]));
      }
      if (k >= a.k || (a.accumulate && !t.count)) continue;
      float* to = a.out + (int64_t)(t.group / a.inner) * a.outer_stride + (int64_t)(t.group % a.inner) * a.inner_stride +
                  (int64_t)(t.m + c0) * a.ld_out + k + t.part() * a.part_stride;
#pragma unroll
      for (int c = 0; c < kOwn; c += 16) {
        float* next = to;
        if (a.accumulate) {
#pragma unroll
          for (int i = 0; i < 16; ++i, next += a.ld_out)
            if (c + i < columns) sum[c + i] += *next;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i, to += a.ld_out)
          if (c + i < columns) *to = sum[c + i];
      }
    }
  }
  tear_down<kCtas>(sh, kTmem);
}

// ---- the sums of divided products --------------------------------------------------------------------------------------------
// Where there are fewer tiles than places to compute them and the summed dimension is long, it is divided (parts_of) and the
// parts are added here, the first to the last (20,000 tokens into two matrices of weight gradients: 21.8 us, undivided 86 us;
// 54 tokens with sums over 3,136 columns: 9.5 us, undivided 17 us).
constexpr int kJoinThreads = 256;

// y = the sum of partial [parts][rows][m], rounded; zeros in rows of no group.
template <typename T>
__global__ void __launch_bounds__(kJoinThreads) k_join_rows(const RowsArgs a) {
  begin_after_predecessor();
  const int64_t head = limited(a.offsets[0], a.rows), tail = limited(a.offsets[a.groups], a.rows), all = (int64_t)a.rows * a.m;
  for (int64_t i = (int64_t)blockIdx.x * kJoinThreads + threadIdx.x; i < all; i += (int64_t)gridDim.x * kJoinThreads) {
    const int64_t row = all >> 32 ? i / a.m : (u32)i / (u32)a.m;
    float s = 0.0f;
    if (row >= head && row < tail) {
#pragma unroll 4
      for (int p = 0; p < a.parts; ++p) s += a.partial[p * all + i];
    }
    static_cast<T*>(a.y)[row * a.ldy + (i - row * a.m)] = from_float<T>(s);
  }
}

// out (+)= the sum of the parts of each group's matrix; `a` describes out, parts those [parts][groups][m][k].
__global__ void __launch_bounds__(kJoinThreads) k_join_weights(const WeightsArgs a, const float* parts) {
  begin_after_predecessor();
  const int64_t matrix = (int64_t)a.m * a.k, all = matrix * a.groups;
  for (int64_t i = (int64_t)blockIdx.x * kJoinThreads + threadIdx.x; i < all; i += (int64_t)gridDim.x * kJoinThreads) {
    const int64_t line = all >> 32 ? i / a.k : (u32)i / (u32)a.k, g = all >> 32 ? line / a.m : (u32)line / (u32)a.m;
    float s = 0.0f;
#pragma unroll 4
    for (int p = 0; p < a.parts; ++p) s += parts[p * all + i];
    float* to = a.out + g / a.inner * a.outer_stride + g % a.inner * a.inner_stride + (line - g * a.m) * a.ld_out + (i - line * a.k);
    *to = a.accumulate ? *to + s : s;
  }
}

// ---- copies of operands that TMA cannot read -------------------------------------------------------------------------------
struct CopyArgs {
  const char* from;
  uint4* to;
  int64_t pitch, stride;    // bytes from line to line and from matrix to matrix
  int64_t lines, total;     // lines of a matrix and of all
  int cols, words;          // of a line: elements, 16-byte words of the copy
};
// The second's work begins at block `blocks`.  Matrices number `skips` holds (the first or the second operand's, or none's) are
// copied only if one of their groups has rows.
struct CopyBoth {
  CopyArgs c[2];
  unsigned blocks;
  int skips, groups, weights;
  const int64_t* offsets;
};

// A thread writes one word of eight elements from the two aligned words that hold them, shifted together.  Those at the ends of
// a line may hold bytes of others, which belong to the same allocation; they land past the columns, where nobody looks.
// Without it TMA could not address such operands at all: its strides are multiples of 16 bytes.  5,003 tokens, 1,030 -> 777 columns of
// float16 over six matrices: 31 us with the copy.
constexpr int kCopyThreads = 256;
__global__ void __launch_bounds__(kCopyThreads) k_copy(const __grid_constant__ CopyBoth both) {
  const bool second = blockIdx.x >= both.blocks;
  const CopyArgs& a = both.c[second];
  const unsigned block = blockIdx.x - (second ? both.blocks : 0), blocks = second ? gridDim.x - both.blocks : both.blocks;
  const int64_t all = a.total * a.words, step = (int64_t)blocks * kCopyThreads;
  __shared__ u32 used[kTableGroups / 32];
  begin_after_predecessor();
  const bool skips = both.skips == (int)second && both.weights > 1;
  if (skips) {
    for (int i = threadIdx.x; i < kTableGroups / 32; i += kCopyThreads) used[i] = 0;
    __syncthreads();
    for (int g = threadIdx.x; g < both.groups; g += kCopyThreads)
      if (both.offsets[g] < both.offsets[g + 1]) atomicOr(&used[g % both.weights / 32], 1u << g % both.weights % 32);
    __syncthreads();
  }
  for (int64_t at = (int64_t)block * kCopyThreads + threadIdx.x; at < all; at += step) {
    const int64_t line = all >> 32 ? at / a.words : (u32)at / (u32)a.words;
    const int word = (int)(at - line * a.words);
    const int64_t matrix = a.total == a.lines ? 0 : a.total >> 31 ? line / a.lines : (u32)line / (u32)a.lines;
    if (skips && !(used[matrix / 32] >> matrix % 32 & 1)) continue;
    const char* p = a.from + matrix * a.stride + (line - matrix * a.lines) * a.pitch + word * 16;
    const u32 skip = (u32)(uintptr_t)p & 15u;  // even
    const uint4* q = reinterpret_cast<const uint4*>(p - skip);
    const uint4 lo = q[0], hi = 16 - (int)skip < min(16, (a.cols - word * 8) * 2) ? q[1] : make_uint4(0, 0, 0, 0);
    u32 w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    if (skip & 8) w[0] = w[2], w[1] = w[3], w[2] = w[4], w[3] = w[5], w[4] = w[6], w[5] = w[7];
    if (skip & 4) w[0] = w[1], w[1] = w[2], w[2] = w[3], w[3] = w[4], w[4] = w[5];
    const u32 shift = (skip & 2) * 8;
    a.to[at] = make_uint4(__funnelshift_r(w[0], w[1], shift), __funnelshift_r(w[1], w[2], shift),
                          __funnelshift_r(w[2], w[3], shift), __funnelshift_r(w[3], w[4], shift));
  }
}

// ---- host --------------------------------------------------------------------------------------------------------------------
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encoder() {
  static EncodeTiled known = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      f = nullptr;
    }
    return reinterpret_cast<EncodeTiled>(f);
  }();
  return known;
}

// Matrices [count][lines][cols] of 16-bit elements, copied in boxes of 64 columns and `box_lines` lines.  count 0: one matrix, 2-D.
bool make_map(CUtensorMap* map, const void* p, int32_t type, int64_t cols, int64_t lines, int64_t ld, int count, int64_t stride, int box_lines) {
  const EncodeTiled encode = encoder();
  if (!encode) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)lines, (cuuint64_t)(count ? count : 1)};
  // one line, one matrix: the distance to the next is never used, but has to be one that is allowed
  cuuint64_t strides[2] = {(cuuint64_t)(lines > 1 ? ld * 2 : (cols * 2 + 15) / 16 * 16), (cuuint64_t)(count > 1 ? stride * 2 : 0)};
  if (count <= 1) strides[1] = strides[0] * dims[1];
  const cuuint32_t box[3] = {kBox, (cuuint32_t)box_lines, 1}, ones[3] = {1, 1, 1};
  return encode(map, type == REGTOPK_TYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, count ? 3 : 2,
                const_cast<void*>(p), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Whether TMA can read the matrices where they are; if not, their copy has lines of round_up(cols, 8) elements.
bool direct(const void* p, int64_t ld, int64_t lines, int count, int64_t stride) {
  return (uintptr_t)p % 16 == 0 && (lines <= 1 || ld % 8 == 0) && (count <= 1 || stride % 8 == 0);
}
int64_t padded(int64_t cols) { return (cols + 7) / 8 * 8; }
size_t copy_bytes(int64_t lines, int64_t cols, int count) { return ((size_t)lines * count * padded(cols) * 2 + 255) / 256 * 256; }

// Operands to copy into the workspace, and their copies.
struct Copies {
  CopyBoth both;
  int count = 0;
  char* ws;
  // Makes p, ld and stride describe the copy.
  void add(const void** p, int64_t* ld, int64_t lines, int64_t cols, int matrices, int64_t* stride) {
    CopyArgs& c = both.c[count++];
    c.from = static_cast<const char*>(*p); c.to = reinterpret_cast<uint4*>(ws); c.pitch = *ld * 2; c.stride = *stride * 2;
    c.lines = lines; c.total = lines * matrices; c.cols = (int)cols; c.words = (int)(padded(cols) / 8);
    *p = ws;
    ws += copy_bytes(lines, cols, matrices);
    *ld = padded(cols);
    *stride = lines * *ld;
  }
  // weights > 1: the operand added last is that many matrices, for the groups of `offsets`.
  int run(const int64_t* offsets, int groups, int weights, int sms, cudaStream_t s) {
    if (!count) return REGTOPK_OK;
    both.skips = count - 1;
    both.offsets = offsets;
    both.groups = groups;
    both.weights = weights;
    unsigned blocks[2] = {0, 0};
    for (int i = 0; i < count; ++i) {
      const int64_t n = (both.c[i].total * both.c[i].words + kCopyThreads - 1) / kCopyThreads, most = (int64_t)sms * 16;
      blocks[i] = (unsigned)(n < most ? n : most);
    }
    both.blocks = blocks[0];
    if (count == 1) both.c[1] = both.c[0];
    return start(k_copy, blocks[0] + blocks[1], kCopyThreads, 0, s, both);
  }
};

template <auto kKernel> bool allow_smem(int bytes, int dev) {
  static uint64_t done;  // of this kernel, one bit a device
  if (__atomic_load_n(&done, __ATOMIC_RELAXED) >> dev & 1) return true;
  if (cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
  __atomic_fetch_or(&done, 1ull << dev, __ATOMIC_RELAXED);
  return true;
}

// Blocks for `tiles` tiles, one for each SM at most; in pairs if a tile is a pair's.
template <int kCtas, typename K, typename... Args>
int launch(K kernel, int64_t tiles, int threads, int smem, int sms, cudaStream_t s, const Args&... args) {
  const int64_t most = sms / kCtas;
  return start<kCtas>(kernel, (unsigned)(tiles < most ? tiles : most) * kCtas, threads, smem, s, args...);
}

template <typename T, int kMost, bool kTransposed, int kCtas, bool kLong>
int launch_rows(const CUtensorMap& w, const CUtensorMap& x, const RowsArgs& a, int64_t token_tiles, int dev, int sms, cudaStream_t s) {
  constexpr auto k = k_rows<T, kMost, kTransposed, kCtas, kLong>;
  constexpr int smem = RowStage<kMost, kCtas>::kSmem;
  if (!allow_smem<k>(smem, dev)) return train_rc(cudaGetLastError());
  return launch<kCtas>(k, token_tiles * ((a.m + kCtas * kLanes - 1) / (kCtas * kLanes)) * a.parts, kRowThreadsOf<kLong>, smem, sms, s, w, x, a);
}

template <typename T, int kCtas>
int launch_weights(const CUtensorMap& x, const CUtensorMap& dy, const WeightsArgs& a, int dev, int sms, cudaStream_t s) {
  constexpr auto k = k_weights<T, kCtas>;
  if (!allow_smem<k>(WeightStage<kCtas>::kSmem, dev)) return train_rc(cudaGetLastError());
  const int64_t tiles = (int64_t)a.groups * ((a.k + kCtas * kLanes - 1) / (kCtas * kLanes)) * ((a.m + kWeightsMost - 1) / kWeightsMost) * a.parts;
  return launch<kCtas>(k, tiles, kWeightThreads, WeightStage<kCtas>::kSmem, sms, s, x, dy, a);
}

// Into how many parts the summed dimension is divided: as many as there are places for (those of 148 SMs, whatever the device has,
// since the workspace's size is asked for without one), but none shorter than 512.  One: not divided.
int parts_of(int64_t tiles, int64_t places, int64_t summed) {
  const int64_t most = tiles > 0 ? places / tiles : 1, parts = summed / 512;
  return (int)(parts < most ? (parts < 1 ? 1 : parts) : most < 1 ? 1 : most);
}
constexpr int kPlaces = 148;

// Coordinates of a copy are 32-bit, and what is worked out from them may pass the end: a tile by 256, an accumulator's terms by kRowsChain,
// a divided dimension by kDepth for each of kPlaces parts.
constexpr int64_t kMostRows = REGTOPK_MATMUL_MAX_SIZE;
static_assert(kMostRows + kRowsChain + kWeightsChain + (int64_t)kPlaces * kDepth < ((int64_t)1 << 31) - 1, "32-bit arithmetic");

struct RowPlan {
  int most, parts, part_k;  // tokens of a tile; parts of the summed dimension and their length
  int64_t tiles;            // of tokens, at most
};

bool good_sizes(int64_t rows, int64_t k, int64_t m, int32_t groups) {
  return rows >= 0 && k >= 0 && m >= 0 && rows <= kMostRows && k <= kMostRows && m <= kMostRows && groups >= 1;
}
// Whether no element of [outer][inner][m] rows of k elements lies in two of them: each distance passes what the smaller ones span.
// Blocks write (and add to) rows on their own, so that rows that overlap would be a race.
bool rows_apart(int64_t k, int64_t m, int64_t ld, int64_t inner, int64_t inner_stride, int64_t outer, int64_t outer_stride) {
  struct { int64_t count, stride; } d[3] = {{m, ld}, {inner, inner_stride}, {outer, outer_stride}};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (d[j].stride > d[j + 1].stride) std::swap(d[j], d[j + 1]);
  __int128 span = k;
  for (const auto& e : d) {
    if (e.count <= 1) continue;
    if (e.stride < span) return false;
    span += (__int128)(e.count - 1) * e.stride;
  }
  return true;
}
bool is_short(int32_t type) { return type == REGTOPK_TYPE_BF16 || type == REGTOPK_TYPE_F16; }

}  // namespace

extern "C" {

static RowPlan row_plan(int64_t rows, int32_t groups, int64_t k, int64_t m) {
  // The widest tile of tokens: as wide as a group has rows on average (a narrower one reads the weights again for nothing, a
  // wider one holds fewer stages); pairs of blocks where they have 256 features to share.
  RowPlan p;
  const int64_t average = rows / groups;
  p.most = average > 64 ? (m > kLanes ? 256 : 128) : average > 32 ? 64 : 32;
  const int ctas = p.most == 256 ? 2 : 1;
  p.tiles = rows / p.most + groups;
  const int64_t all = p.tiles * ((m + ctas * kLanes - 1) / (ctas * kLanes));
  p.parts = k >= 2048 ? parts_of(all, kPlaces / ctas, k) : 1;
  p.part_k = p.parts > 1 ? (int)((k + p.parts - 1) / p.parts + kDepth - 1) / kDepth * kDepth : (int)k;
  if (p.parts > 1) p.parts = (int)((k + p.part_k - 1) / p.part_k);
  return p;
}
static size_t partial_bytes(int parts, int64_t elements) { return parts > 1 ? ((size_t)parts * elements * 4 + 255) / 256 * 256 : 0; }
static int weight_parts(int64_t rows, int32_t groups, int64_t k, int64_t m) {
  const int ctas = k > kLanes ? 2 : 1;
  return parts_of(groups * ((k + ctas * kLanes - 1) / (ctas * kLanes)) * ((m + kWeightsMost - 1) / kWeightsMost), kPlaces / ctas, rows / groups);
}

size_t regtopk_grouped_matmul_workspace_bytes(const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t w_stride,
                                              int32_t transposed, int32_t weights, int32_t groups, int64_t rows, int64_t k,
                                              int64_t m) {
  if (!good_sizes(rows, k, m, groups) || weights < 1) return 0;
  const int64_t lines = transposed ? k : m, cols = transposed ? m : k;
  const int count = w_stride ? weights : 1;
  return (direct(x, ldx, rows, 1, 0) ? 0 : copy_bytes(rows, k, 1)) + (direct(w, ldw, lines, count, w_stride) ? 0 : copy_bytes(lines, cols, count)) +
         partial_bytes(row_plan(rows, groups, k, m).parts, rows * m);
}

int regtopk_grouped_matmul(const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t w_stride, int32_t transposed,
                           int32_t weights, void* y, int64_t ldy, const int64_t* offsets, int32_t groups, int64_t rows,
                           int64_t k, int64_t m, int32_t type, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!is_short(type) || !good_sizes(rows, k, m, groups) || weights < 1 || groups % weights || !offsets || (uintptr_t)offsets % 8 || w_stride < 0)
    return REGTOPK_ERR_INVALID_ARG;
  if (groups > REGTOPK_MATMUL_MAX_GROUPS) return REGTOPK_ERR_TOO_LARGE;
  if (rows == 0 || m == 0) return REGTOPK_OK;
  int64_t lines = transposed ? k : m, cols = transposed ? m : k;
  if (!good_matrix(y, ldy, rows, m, 2)) return REGTOPK_ERR_INVALID_ARG;
  if (k > 0 && (!good_matrix(x, ldx, rows, k, 2) || !good_matrix(w, ldw, lines, cols, 2))) return REGTOPK_ERR_INVALID_ARG;
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (k == 0) return train_rc(cudaMemset2DAsync(y, (size_t)(rows > 1 ? ldy : m) * 2, 0, (size_t)m * 2, (size_t)rows, s));
  const size_t need = regtopk_grouped_matmul_workspace_bytes(x, ldx, w, ldw, w_stride, transposed, weights, groups, rows, k, m);
  if (need && (!workspace || (uintptr_t)workspace % 16)) return REGTOPK_ERR_INVALID_ARG;
  if (workspace_bytes < need) return REGTOPK_ERR_WORKSPACE_TOO_SMALL;
  const int count = w_stride ? weights : 1;
  int64_t none = 0;
  Copies copies;
  copies.ws = static_cast<char*>(workspace);
  if (!direct(x, ldx, rows, 1, 0)) copies.add(&x, &ldx, rows, k, 1, &none);
  const bool copies_w = !direct(w, ldw, lines, count, w_stride);
  if (copies_w) copies.add(&w, &ldw, lines, cols, count, &w_stride);
  const int rc = copies.run(offsets, groups, copies_w ? count : 1, sms, s);
  if (rc != REGTOPK_OK) return rc;

  const RowPlan plan = row_plan(rows, groups, k, m);
  const int most = plan.most;
  CUtensorMap wm, xm;
  if (!make_map(&wm, w, type, cols, lines, ldw, count, w_stride, transposed ? kDepth : kLanes) ||
      !make_map(&xm, x, type, k, rows, ldx, 0, 0, most < 64 ? most : 64)) return REGTOPK_ERR_CUDA;
  RowsArgs a;
  a.offsets = offsets; a.y = y; a.ldy = ldy; a.groups = groups; a.weights = weights; a.rows = (int)rows; a.k = (int)k; a.m = (int)m;
  a.shared_weights = count == 1;
  a.pairs = m % 2 == 0 && (rows == 1 || ldy % 2 == 0) && (uintptr_t)y % 4 == 0;
  a.parts = plan.parts; a.part_k = plan.part_k; a.partial = reinterpret_cast<float*>(copies.ws);
  const int64_t tiles = plan.tiles;
  if (tiles * ((m + kLanes - 1) / kLanes) > INT32_MAX) return REGTOPK_ERR_TOO_LARGE;
  auto launch_product = [&]() -> int {
#define REGTOPK_ROWS(N, C, L)                                                                        \
  return type == REGTOPK_TYPE_BF16                                                                   \
             ? (transposed ? launch_rows<__nv_bfloat16, N, true, C, L>(wm, xm, a, tiles, dev, sms, s)  \
                           : launch_rows<__nv_bfloat16, N, false, C, L>(wm, xm, a, tiles, dev, sms, s)) \
             : (transposed ? launch_rows<__half, N, true, C, L>(wm, xm, a, tiles, dev, sms, s)         \
                           : launch_rows<__half, N, false, C, L>(wm, xm, a, tiles, dev, sms, s))
#define REGTOPK_ROWS_OF(N, C)               \
  if (a.part_k > kRowsChain) REGTOPK_ROWS(N, C, true); \
  REGTOPK_ROWS(N, C, false)
    switch (most) {
      case 32: REGTOPK_ROWS_OF(32, 1);
      case 64: REGTOPK_ROWS_OF(64, 1);
      case 128: REGTOPK_ROWS_OF(128, 1);
      default: REGTOPK_ROWS_OF(256, 2);
    }
#undef REGTOPK_ROWS_OF
#undef REGTOPK_ROWS
  };
  const int done = launch_product();
  if (done != REGTOPK_OK || a.parts == 1) return done;
  const int64_t blocks = (rows * m + kJoinThreads - 1) / kJoinThreads, most_blocks = (int64_t)sms * 8;
  const dim3 grid((unsigned)(blocks < most_blocks ? blocks : most_blocks));
  return type == REGTOPK_TYPE_BF16 ? start(k_join_rows<__nv_bfloat16>, grid, kJoinThreads, 0, s, a)
                                   : start(k_join_rows<__half>, grid, kJoinThreads, 0, s, a);
}

size_t regtopk_grouped_matmul_dw_workspace_bytes(const void* dy, int64_t ld_dy, const void* x, int64_t ldx, int32_t groups,
                                                 int64_t rows, int64_t k, int64_t m) {
  if (!good_sizes(rows, k, m, groups)) return 0;
  return (direct(dy, ld_dy, rows, 1, 0) ? 0 : copy_bytes(rows, m, 1)) + (direct(x, ldx, rows, 1, 0) ? 0 : copy_bytes(rows, k, 1)) +
         partial_bytes(weight_parts(rows, groups, k, m), groups * m * k);
}

int regtopk_grouped_matmul_dw(const void* dy, int64_t ld_dy, const void* x, int64_t ldx, float* out, int64_t ld_out,
                              int64_t inner_stride, int64_t outer_stride, int32_t inner, int32_t accumulate,
                              const int64_t* offsets, int32_t groups, int64_t rows, int64_t k, int64_t m, int32_t type,
                              void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!is_short(type) || !good_sizes(rows, k, m, groups) || inner < 1 || groups % inner || !offsets || (uintptr_t)offsets % 8 ||
      inner_stride < 0 || outer_stride < 0) return REGTOPK_ERR_INVALID_ARG;
  if (groups > REGTOPK_MATMUL_MAX_GROUPS) return REGTOPK_ERR_TOO_LARGE;
  if (k == 0 || m == 0) return REGTOPK_OK;
  if (!good_matrix(out, ld_out, m, k, 4) || !rows_apart(k, m, ld_out, inner, inner_stride, groups / inner, outer_stride)) return REGTOPK_ERR_INVALID_ARG;
  if (rows > 0 && (!good_matrix(dy, ld_dy, rows, m, 2) || !good_matrix(x, ldx, rows, k, 2))) return REGTOPK_ERR_INVALID_ARG;
  if (rows == 0 && accumulate) return REGTOPK_OK;
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  WeightsArgs a;
  float* partial = nullptr;
  CUtensorMap xm, ym;
  if (rows > 0) {
    const size_t need = regtopk_grouped_matmul_dw_workspace_bytes(dy, ld_dy, x, ldx, groups, rows, k, m);
    if (need && (!workspace || (uintptr_t)workspace % 16)) return REGTOPK_ERR_INVALID_ARG;
    if (workspace_bytes < need) return REGTOPK_ERR_WORKSPACE_TOO_SMALL;
    int64_t none = 0;
    Copies copies;
    copies.ws = static_cast<char*>(workspace);
    if (!direct(dy, ld_dy, rows, 1, 0)) copies.add(&dy, &ld_dy, rows, m, 1, &none);
    if (!direct(x, ldx, rows, 1, 0)) copies.add(&x, &ldx, rows, k, 1, &none);
    const int rc = copies.run(offsets, groups, 1, sms, s);
    if (rc != REGTOPK_OK) return rc;
    partial = reinterpret_cast<float*>(copies.ws);
    if (!make_map(&xm, x, type, k, rows, ldx, 0, 0, kDepth) || !make_map(&ym, dy, type, m, rows, ld_dy, 0, 0, kDepth)) return REGTOPK_ERR_CUDA;
  } else {
    memset(&xm, 0, sizeof xm);  // never used: no group has rows
    memset(&ym, 0, sizeof ym);
  }
  a.offsets = offsets; a.out = out; a.ld_out = ld_out; a.inner_stride = inner_stride; a.outer_stride = outer_stride;
  a.groups = groups; a.inner = inner; a.rows = (int)rows; a.k = (int)k; a.m = (int)m; a.accumulate = accumulate;
  if ((k + kLanes - 1) / kLanes * ((m + kWeightsMost - 1) / kWeightsMost) * groups > INT32_MAX) return REGTOPK_ERR_TOO_LARGE;
  a.parts = rows > 0 ? weight_parts(rows, groups, k, m) : 1;
  a.part_stride = (int64_t)groups * m * k;
  const bool pairs = k > kLanes;
  const auto product = [&](const WeightsArgs& p) {
    if (type == REGTOPK_TYPE_BF16)
      return pairs ? launch_weights<__nv_bfloat16, 2>(xm, ym, p, dev, sms, s) : launch_weights<__nv_bfloat16, 1>(xm, ym, p, dev, sms, s);
    return pairs ? launch_weights<__half, 2>(xm, ym, p, dev, sms, s) : launch_weights<__half, 1>(xm, ym, p, dev, sms, s);
  };
  if (a.parts == 1) return product(a);
  WeightsArgs p = a;  // into the workspace
  p.out = partial; p.ld_out = k; p.inner = groups; p.inner_stride = m * k; p.outer_stride = 0; p.accumulate = 0;
  const int rc = product(p);
  if (rc != REGTOPK_OK) return rc;
  const int64_t blocks = (a.part_stride + kJoinThreads - 1) / kJoinThreads, most = (int64_t)sms * 8;
  return start(k_join_weights, dim3((unsigned)(blocks < most ? blocks : most)), kJoinThreads, 0, s, a, partial);
}

int regtopk_train_status(void* cuda_stream) {
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  int rc = gave_up(s);
  if (rc == 0) rc = regtopk_norm_gave_up(s);
  if (rc == 0) rc = regtopk_rms_gave_up(s);
  return rc > 0 ? REGTOPK_ERR_INTERNAL : rc;
}

}  // extern "C"
