// The router: the choice of experts with its weights and their gradient, and the order of (worker, expert) groups
// (include/regtopk_experts.h).
//
// A token's logits are a few hundred numbers, so that a warp keeps them in registers and chooses by comparing there; the logits are
// read once.  What bounds the choice is the issue of instructions, some 300 of a warp for eight of 256 experts, not the memory.

#include <float.h>

#include "rows8.cuh"

namespace {

constexpr int kRouteThreads = 256, kRouteWarps = kRouteThreads / 32;

struct RouteArgs {
  const void* logits;
  const float* bias;
  int32_t* experts;
  float* weights;
  int64_t ld, tokens;
  int n_experts, k;
  int groups, size, kept, top;    // size: experts of a group
  int lanes_log2, lanes, each;    // lanes of a group, experts of a lane (at most the template's N)
  int wide;                       // every lane has N neighbours, aligned, or none
  int sigmoid, renormalise;
  float scale;
};

// Binary32 numbers as whole numbers of the same order (-0 as +0).  0 is left for what cannot be chosen, and NaN is below all numbers.
__device__ __forceinline__ u32 ordered(float v) {
  const u32 b = __float_as_uint(v + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(u32 o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
  return v;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}

// A lane's experts: N neighbours of one group (fewer at its end), so that lanes, and elements in a lane, ascend with the experts.
struct Share {
  int group, first, count;
  __device__ __forceinline__ Share(const RouteArgs& a, int lane) {
    group = lane >> a.lanes_log2;
    const int within = (lane & (a.lanes - 1)) * a.each;
    first = group * a.size + within;
    count = group < a.groups ? min(a.each, a.size - within) : 0;
  }
};

template <typename T, int N> __device__ __forceinline__ void read_logits(float (&l)[N], const T* row, const Share& own, int wide) {
  constexpr int kBytes = N * (int)sizeof(T);
  if (kBytes >= 4 && wide) {
    T v[N];
    if (own.count > 0) {
      const T* p = row + own.first;
      if constexpr (kBytes == 4) *reinterpret_cast<u32*>(v) = *reinterpret_cast<const u32*>(p);
      if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(v) = *reinterpret_cast<const uint2*>(p);
      if constexpr (kBytes >= 16) {
#pragma unroll
        for (int i = 0; i < kBytes / 16; ++i) reinterpret_cast<uint4*>(v)[i] = reinterpret_cast<const uint4*>(p)[i];
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) l[i] = own.count > 0 ? to_float(v[i]) : -INFINITY;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) l[i] = i < own.count ? to_float(row[own.first + i]) : -INFINITY;
  }
}

// The choice in binary64, for the few tokens whose numbers lie too close for binary32: into slots[0 .. k), as many as it returns.
// `by_logit`: the experts are compared by their logits, which are exact.
template <typename T, int N>
__device__ __noinline__ int choose_in_64_bits(const RouteArgs& a, const T* row, int* slots, int lane) {
  const Share own(a, lane);
  double c[N], most = -INFINITY;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    c[i] = i < own.count ? (double)to_float(row[own.first + i]) : -INFINITY;
    if (c[i] > most) most = c[i];
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) most = fmax(most, __shfl_xor_sync(kAll, most, o));
  double total = 0.0;
  if (!a.sigmoid) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (c[i] != -INFINITY) total += exp(c[i] - most);
    total = warp_sum(total);
  }
  const bool scores = a.bias || a.top == 2;
  double t1 = -INFINITY, t2 = -INFINITY;  // of this lane, then of its group
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (c[i] == -INFINITY) continue;
    double s = c[i];
    if (scores) {
      s = a.sigmoid ? 1.0 / (1.0 + exp(-s)) : exp(s - most) / total;
      if (a.bias) s += (double)a.bias[own.first + i];
    }
    if (s != s) s = -DBL_MAX;
    if (a.bias || c[i] != c[i]) c[i] = s != -INFINITY ? (c[i] != c[i] ? -DBL_MAX : s) : -INFINITY;
    if (s > t1) {
      t2 = t1;
      t1 = s;
    } else if (s > t2) {
      t2 = s;
    }
  }
  if (a.groups > 1) {
    for (int o = 1; o < a.lanes; o <<= 1) {
      const double o1 = __shfl_xor_sync(kAll, t1, o), o2 = __shfl_xor_sync(kAll, t2, o);
      t2 = fmax(fmin(t1, o1), fmax(t2, o2));
      t1 = fmax(t1, o1);
    }
    const double strength = a.top == 2 && t2 != -INFINITY ? t1 + t2 : t1;
    int rank = 0;
    for (int g = 0; g < a.groups; ++g) {
      const double s = __shfl_sync(kAll, strength, g << a.lanes_log2);
      rank += s > strength || (s == strength && g < own.group);
    }
    if (rank >= a.kept) {
#pragma unroll
      for (int i = 0; i < N; ++i) c[i] = -INFINITY;
    }
  }
  for (int j = 0; j < a.k; ++j) {
    double best = -INFINITY;
    int e = INT32_MAX;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (c[i] > best) {
        best = c[i];
        e = own.first + i;
      }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      const double b = __shfl_xor_sync(kAll, best, o);
      const int f = __shfl_xor_sync(kAll, e, o);
      if (b > best || (b == best && f < e)) {
        best = b;
        e = f;
      }
    }
    if (best == -INFINITY) return j;
    if (lane == 0) slots[j] = e;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (own.first + i == e && i < own.count) c[i] = -INFINITY;
  }
  return a.k;
}

// Descending order within a lane (Batcher's odd-even merge sort).
template <int N> __device__ __forceinline__ void sort_descending(u32 (&v)[N]) {
#pragma unroll
  for (int p = 1; p < N; p *= 2)
#pragma unroll
    for (int q = p; q >= 1; q /= 2)
#pragma unroll
      for (int j = q % p; j + q < N; j += 2 * q)
#pragma unroll
        for (int i = 0; i < q; ++i)
          if (i + j + q < N && (i + j) / (2 * p) == (i + j + q) / (2 * p)) {
            const u32 x = v[i + j], y = v[i + j + q];
            v[i + j] = max(x, y);
            v[i + j + q] = min(x, y);
          }
}

// The weights of the experts chosen, one a lane, as shares: exp(l) (softmax) or 1 / (1 + exp(-l)) over their sum.  Everything is
// taken relative to the largest, so that no sum is 0 whatever the logits.
__device__ __forceinline__ float share_of(float l, bool there, bool sigmoid) {
  float most = warp_max(there ? l : -INFINITY), v;
  if (sigmoid) {
    most = fminf(most, 0.0f);
    v = l < 0.0f ? expf(l - most) / (1.0f + expf(l)) : 1.0f / (1.0f + expf(-l));
  } else {
    v = expf(l - most);
  }
  if (!there) v = 0.0f;
  return v / warp_sum(v);
}

// A token's experts are found by k times taking the largest key of the warp.  A key is a number in the order of c (of the logits
// themselves without bias: the order is the same) whose low bits say which of the lane's experts it belongs to, so that one
// reduction finds number and place.
//   16-bit logits, no bias: the low bits of the numbers are 0, the expert's own number fits there, and the keys are in the exact
//   order, ties included.
//   Otherwise log2(N) bits are cut off and the scores themselves are rounded: tokens among whose first k + 1 numbers, or
//   groups, two are closer than both errors together go to choose_in_64_bits.
// Errors: an expf within 2 units of its last place and the rounding of its argument x, which changes x exp(-x) by 0.37 units of
// 2^-24 at most; a sum of up to 512 of them as a tree of at most 21 additions; a division: 2^-19 of the largest score covers them.
template <typename T, int N>
__global__ void __launch_bounds__(kRouteThreads) k_route(const __grid_constant__ RouteArgs a) {
  __shared__ int all_slots[kRouteWarps][REGTOPK_ROUTE_MAX_CHOICES];
  begin_after_predecessor();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int* slots = all_slots[warp];
  const Share own(a, lane);
  float bias[N];
#pragma unroll
  for (int i = 0; i < N; ++i) bias[i] = a.bias && i < own.count ? a.bias[own.first + i] : 0.0f;
  const bool scored = a.bias || (a.groups > 1 && a.top == 2), exact_keys = sizeof(T) == 2 && !a.bias;
  const int64_t step = (int64_t)gridDim.x * kRouteWarps;
  for (int64_t t = (int64_t)blockIdx.x * kRouteWarps + warp; t < a.tokens; t += step) {
    const T* row = static_cast<const T*>(a.logits) + t * a.ld;
    float l[N];
    read_logits<T, N>(l, row, own, a.wide);
    // softmax: the largest logit, the sum of all exponentials beside it
    bool bad = false;
    float most = -INFINITY, total = 1.0f, per_total = 1.0f;
    if (!a.sigmoid) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        most = fmaxf(most, l[i]);
        bad |= !(l[i] <= FLT_MAX);
      }
      bad = __any_sync(kAll, bad);
      if (scored || !a.renormalise) {
        most = warp_max(most);
        total = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) total += l[i] == -INFINITY ? 0.0f : expf(l[i] - most);
        total = warp_sum(total);
        per_total = 1.0f / total;
      }
    }
    const float margin = scored ? 0x1p-18f * per_total : 0.0f;  // of the difference of two scores
    bool near = false;
    u32 key[N];
    float t1 = -INFINITY, t2 = -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float c = l[i], s = l[i];
      if (scored) {
        s = a.sigmoid ? __fdividef(1.0f, 1.0f + __expf(-c)) : expf(c - most) * per_total;
        if (a.bias) c = s = s + bias[i];
        if (l[i] == -INFINITY) c = s = -INFINITY;
      }
      if (s != s) s = -FLT_MAX;
      t2 = fmaxf(t2, fminf(t1, s));
      t1 = fmaxf(t1, s);
      const u32 low = exact_keys ? 511u - (u32)(own.first + i) : (u32)(N - 1 - i), mask = exact_keys ? 511u : (u32)(N - 1);
      key[i] = c == -INFINITY ? 0u : c != c ? 0x400u | low : (ordered(c) & ~mask) | low;
    }
    if (a.groups > 1) {
      for (int o = 1; o < a.lanes; o <<= 1) {
        const float o1 = __shfl_xor_sync(kAll, t1, o), o2 = __shfl_xor_sync(kAll, t2, o);
        t2 = fmaxf(fminf(t1, o1), fmaxf(t2, o2));
        t1 = fmaxf(t1, o1);
      }
      const float strength = a.top == 2 && t2 != -INFINITY ? t1 + t2 : t1;
      int rank = 0;
      for (int g = 0; g < a.groups; ++g) {
        const float s = __shfl_sync(kAll, strength, g << a.lanes_log2);
        rank += s > strength || (s == strength && g < own.group);
        near |= scored && g != own.group && own.group < a.groups && fabsf(s - strength) <= fmaf(0x1p-21f, fabsf(s) + fabsf(strength), 2.0f * margin);
      }
      if (rank >= a.kept) {
#pragma unroll
        for (int i = 0; i < N; ++i) key[i] = 0;
      }
    }
    // the k largest keys
    constexpr bool kSorted = N <= 8;
    if (kSorted) sort_descending<N>(key);
    u32 mine = 0, beyond = 0;  // lane j: the j-th largest; beyond: the one after the last
    int picked = 0;
    for (int j = 0;; ++j) {
      u32 top = key[0];
      if (!kSorted) {
#pragma unroll
        for (int i = 1; i < N; ++i) top = max(top, key[i]);
      }
      const u32 m = __reduce_max_sync(kAll, top);
      if (j == a.k) {
        beyond = m;
        break;
      }
      if (m == 0) break;
      ++picked;
      if (lane == j) mine = m;
      const u32 holders = __ballot_sync(kAll, top == m);
      near |= (holders & (holders - 1)) != 0;  // never among exact keys
      if (top == m) {
        slots[j] = exact_keys ? (int)(511u - (m & 511u)) : own.first + N - 1 - (int)(m & (N - 1));
        if (kSorted) {
#pragma unroll
          for (int i = 0; i + 1 < N; ++i) key[i] = key[i + 1];
          key[N - 1] = 0;
        } else {
#pragma unroll
          for (int i = 0; i < N; ++i) key[i] = key[i] == m ? 0u : key[i];
        }
      }
    }
    if (!exact_keys) {
      constexpr u32 kMask = N - 1;
      u32 next = __shfl_down_sync(kAll, mine, 1);
      if (lane == picked - 1) next = beyond;
      if (lane < picked && next) {
        const float v = unordered(mine & ~kMask), w = unordered(next & ~kMask);
        near |= !(v - w > fmaf(N * 0x1p-22f, fabsf(v) + fabsf(w), margin)) && v < INFINITY && next > 0x7FFu;
        near |= v == INFINITY && w == INFINITY;
        near |= mine < 0x800u;  // NaN: their order in a lane and over lanes
      }
    }
    __syncwarp();
    if (__any_sync(kAll, near)) picked = choose_in_64_bits<T, N>(a, row, slots, lane);
    __syncwarp();
    const bool there = lane < picked;
    const int e = there ? slots[lane] : -1;
    __syncwarp();
    const float logit = there ? to_float(row[e]) : 0.0f;
    float w;
    if (a.renormalise) w = share_of(logit, there, a.sigmoid);
    else if (a.sigmoid) w = 1.0f / (1.0f + expf(-logit));
    else w = expf(logit - most) / total;
    w = bad ? __uint_as_float(0x7FC00000u) : w * a.scale;
    if (lane < a.k) {
      a.experts[t * a.k + lane] = e;
      a.weights[t * a.k + lane] = there ? w : 0.0f;
    }
  }
}

// ---- the gradient to the logits ------------------------------------------------------------------------------------
struct RouteBackArgs {
  const float* dweights;
  const void* logits;
  const int32_t* experts;
  void* dlogits;
  int64_t ld, ldd, tokens;
  int n_experts, k, wide, sigmoid, renormalise;
  float scale;
};

// A warp a token.  What reaches the chosen experts' scores, or logits, is laid into a row in shared memory, from which the
// gradient row is written.  Plain softmax scores need all logits, the others only the chosen ones.
template <typename T> __global__ void __launch_bounds__(kRouteThreads) k_route_back(const __grid_constant__ RouteBackArgs a) {
  __shared__ float rows[kRouteWarps][REGTOPK_ROUTE_MAX_EXPERTS];
  begin_after_predecessor();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float* own = rows[warp];
  const bool dense = !a.sigmoid && !a.renormalise;
  const int64_t step = (int64_t)gridDim.x * kRouteWarps;
  for (int64_t t = (int64_t)blockIdx.x * kRouteWarps + warp; t < a.tokens; t += step) {
    const T* row = static_cast<const T*>(a.logits) + t * a.ld;
    T* out = static_cast<T*>(a.dlogits) + t * a.ldd;
    int e = lane < a.k ? a.experts[t * a.k + lane] : -1;
    const bool there = e >= 0 && e < a.n_experts;
    const float dw = there ? a.dweights[t * a.k + lane] : 0.0f, l = there ? to_float(row[e]) : 0.0f;
    float most = -INFINITY, per_total = 0.0f, mean = 0.0f, g;
    if (dense) {
      for (int i = lane; i < a.n_experts; i += 32) most = fmaxf(most, to_float(row[i]));
      most = warp_max(most);
      float total = 0.0f;
      for (int i = lane; i < a.n_experts; i += 32) {
        const float v = to_float(row[i]);
        total += v == -INFINITY ? 0.0f : expf(v - most);
      }
      total = warp_sum(total);
      per_total = total > 0.0f ? 1.0f / total : total;  // a row without experts has no scores
      g = a.scale * dw;
      mean = warp_sum(there && l != -INFINITY ? g * expf(l - most) * per_total : 0.0f);
    } else if (a.renormalise) {
      const float p = share_of(l, there, a.sigmoid);
      g = a.scale * p * (dw - warp_sum(there ? dw * p : 0.0f));
      if (a.sigmoid) g /= 1.0f + expf(l);
    } else {
      const float q = expf(-fabsf(l)), r = 1.0f / (1.0f + q);
      g = a.scale * dw * (q * r) * r;
    }
    for (int i = lane; i < a.n_experts; i += 32) own[i] = 0.0f;
    __syncwarp();
    const u32 same = __match_any_sync(kAll, there ? e : -1 - lane);
    if (__any_sync(kAll, there && (same & (same - 1)))) {  // the same expert twice: one after the other, in order
      for (int j = 0; j < a.k; ++j) {
        if (lane == j && there) own[e] += g;
        __syncwarp();
      }
    } else if (there) {
      own[e] = g;
    }
    __syncwarp();
    if (a.wide) {
      for (int i = lane * 8; i < a.n_experts; i += 256) {
        Octet f;
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = reinterpret_cast<const float2*>(own + i)[j];
        if (dense) {
          Eight<T> v;
          Octet x;
          v.fetch(row + i);
          v.get(x);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            f[j].x = x[j].x == -INFINITY ? 0.0f : expf(x[j].x - most) * per_total * (f[j].x - mean);
            f[j].y = x[j].y == -INFINITY ? 0.0f : expf(x[j].y - most) * per_total * (f[j].y - mean);
          }
        }
        Eight<T> v;
        v.put(f);
        v.store(out + i);
      }
    } else {
      for (int i = lane; i < a.n_experts; i += 32) {
        float f = own[i];
        if (dense) {
          const float x = to_float(row[i]);
          f = x == -INFINITY ? 0.0f : expf(x - most) * per_total * (f - mean);
        }
        out[i] = from_float<T>(f);
      }
    }
    __syncwarp();
  }
}

// ---- the order of groups ---------------------------------------------------------------------------------------------
// A counting sort.  The pairs (token, choice), in their order, are cut into chunks, one a block, and a chunk into one run for every
// warp.  Where a pair goes: to the start of its group, past the pairs of the group in the chunks before (k_sort_count has counted
// them), in the runs before and in its own run, which a warp goes through in steps of 32.  Nothing depends on the order in which
// blocks or warps run.  A sort of one chunk is a single launch.
struct SortArgs {
  const int32_t* experts;
  const int64_t* workers_at;  // NULL: all tokens are of worker 0
  int64_t* offsets;
  int32_t* place;
  u32* counts;  // [chunks][groups]
  int64_t tokens, pairs;
  Divisor k;
  int workers, n_experts, groups, chunk, chunks;
};

constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32;

// The group of a pair, or -1.
__device__ __forceinline__ int group_of_pair(const SortArgs& a, u32 pair) {
  const int e = a.experts[pair];
  if (e < 0 || e >= a.n_experts) return -1;
  if (!a.workers_at) return e;
  const int64_t t = a.k.quotient_of(pair);
  if (t < a.workers_at[0] || t >= a.workers_at[a.workers]) return -1;
  int lo = 0, hi = a.workers;  // the last worker that begins at t or before
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.workers_at[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo * a.n_experts + e;
}

__global__ void __launch_bounds__(kSortThreads) k_sort_count(const __grid_constant__ SortArgs a) {
  __shared__ u32 count[REGTOPK_MATMUL_MAX_GROUPS];
  begin_after_predecessor();
  for (int g = threadIdx.x; g < a.groups; g += kSortThreads) count[g] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * a.chunk, end = min(first + a.chunk, a.pairs);
  for (int64_t p = first + threadIdx.x; p < end; p += kSortThreads) {
    const int g = group_of_pair(a, (u32)p);
    if (g >= 0) atomicAdd(&count[g], 1u);
  }
  __syncthreads();
  for (int g = threadIdx.x; g < a.groups; g += kSortThreads) a.counts[(int64_t)blockIdx.x * a.groups + g] = count[g];
}

// dynamic shared memory: base [groups], then runs [warps][groups]
__global__ void __launch_bounds__(kSortThreads) k_sort_place(const __grid_constant__ SortArgs a) {
  extern __shared__ __align__(16) char smem[];
  __shared__ u32 sums[kSortWarps];
  begin_after_predecessor();
  u32* base = reinterpret_cast<u32*>(smem);
  u32* runs = base + a.groups;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int i = threadIdx.x; i < kSortWarps * a.groups; i += kSortThreads) runs[i] = 0;
  __syncthreads();
  // this warp's run
  const int64_t first = (int64_t)blockIdx.x * a.chunk, end = min(first + a.chunk, a.pairs);
  const int64_t length = ((end - first + kSortWarps - 1) / kSortWarps + 31) & ~31ll, from = first + warp * length, to = min(from + length, end);
  u32* own = runs + warp * a.groups;
  for (int64_t p = from + lane; p - lane < to; p += 32) {
    const int g = p < to ? group_of_pair(a, (u32)p) : -1;
    const u32 same = __match_any_sync(kAll, g);
    if (g >= 0 && lane == __ffs(same) - 1) own[g] += __popc(same);
    __syncwarp();
  }
  __syncthreads();
  // of every group: its size, what lies in the chunks before, and within this one in the runs before
  u32 at = 0;  // start of the groups that this round of threads looks at
  for (int g0 = 0; g0 < a.groups; g0 += kSortThreads) {
    const int g = g0 + threadIdx.x;
    u32 total = 0, before = 0;
    if (g < a.groups) {
      u32 here = 0;
      for (int w = 0; w < kSortWarps; ++w) {
        const u32 n = runs[w * a.groups + g];
        runs[w * a.groups + g] = here;
        here += n;
      }
      if (a.chunks == 1) {
        total = here;
      } else {
#pragma unroll 8
        for (int c = 0; c < a.chunks; ++c) {
          const u32 n = a.counts[(int64_t)c * a.groups + g];
          total += n;
          before += c < (int)blockIdx.x ? n : 0;
        }
      }
    }
    u32 scan = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u32 v = __shfl_up_sync(kAll, scan, o);
      if (lane >= o) scan += v;
    }
    if (lane == 31) sums[warp] = scan;
    __syncthreads();
    u32 lower = at, all = at;
    for (int w = 0; w < kSortWarps; ++w) {
      if (w < warp) lower += sums[w];
      all += sums[w];
    }
    if (g < a.groups) {
      base[g] = lower + scan - total + before;
      if (blockIdx.x == 0) {
        a.offsets[g] = lower + scan - total;
        if (g == a.groups - 1) a.offsets[a.groups] = lower + scan;
      }
    }
    at = all;
    __syncthreads();
  }
  for (int64_t p = from + lane; p - lane < to; p += 32) {
    const int g = p < to ? group_of_pair(a, (u32)p) : -1;
    const u32 same = __match_any_sync(kAll, g);
    const u32 rank = __popc(same & ((1u << lane) - 1));
    u32 where = 0;
    if (g >= 0) where = base[g] + own[g] + rank;
    __syncwarp();
    if (g >= 0 && rank == 0) own[g] += __popc(same);
    __syncwarp();
    if (p < to) a.place[p] = g >= 0 ? (int32_t)where : -1;
  }
}

// Pairs of a chunk: see regtopk_sort_tokens.
inline int chunk_of(int64_t pairs) {
  int64_t chunk = pairs <= 4096 ? 4096 : 1024;
  while (chunk * 128 < pairs) chunk *= 2;
  return (int)chunk;
}

template <auto kKernel> bool allow_smem_of(int dev, int bytes) {
  static uint64_t done;  // of this kernel, one bit a device
  if (__atomic_load_n(&done, __ATOMIC_RELAXED) >> dev & 1) return true;
  if (cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
  __atomic_fetch_or(&done, 1ull << dev, __ATOMIC_RELAXED);
  return true;
}

template <typename T, int N> int launch_route(const RouteArgs& a, int sms, cudaStream_t s) {
  const int64_t blocks = (a.tokens + kRouteWarps - 1) / kRouteWarps, most = (int64_t)sms * 8;
  return start(k_route<T, N>, (unsigned)(blocks < most ? blocks : most), kRouteThreads, 0, s, a);
}
template <typename T> int launch_route_of(RouteArgs& a, int sms, cudaStream_t s) {
  int n = 1;
  while (n < a.each) n *= 2;
  const int bytes = n * (int)sizeof(T) < 16 ? n * (int)sizeof(T) : 16;
  a.wide = n == a.each && a.size % n == 0 && (uintptr_t)a.logits % bytes == 0 && (a.tokens <= 1 || a.ld * (int64_t)sizeof(T) % bytes == 0);
  switch (n) {
    case 1: return launch_route<T, 1>(a, sms, s);
    case 2: return launch_route<T, 2>(a, sms, s);
    case 4: return launch_route<T, 4>(a, sms, s);
    case 8: return launch_route<T, 8>(a, sms, s);
    case 16: return launch_route<T, 16>(a, sms, s);
    default: return launch_route<T, 32>(a, sms, s);
  }
}
template <typename T> int launch_route_back(const RouteBackArgs& a, int sms, cudaStream_t s) {
  const int64_t blocks = (a.tokens + kRouteWarps - 1) / kRouteWarps, most = (int64_t)sms * 8;
  return start(k_route_back<T>, (unsigned)(blocks < most ? blocks : most), kRouteThreads, 0, s, a);
}

inline bool good_route(const regtopk_route_params* p, int n_experts) {
  return p && (p->scores == REGTOPK_SCORES_SOFTMAX || p->scores == REGTOPK_SCORES_SIGMOID) && p->groups >= 1 && n_experts % p->groups == 0 &&
         p->groups_kept >= 1 && p->groups_kept <= p->groups && (p->group_top == 1 || p->group_top == 2) && p->scale - p->scale == 0.0f;
}

}  // namespace

extern "C" {

int regtopk_route(const void* logits, int64_t ld_logits, const float* bias, int32_t* experts, float* weights, int64_t tokens,
                  int32_t n_experts, int32_t k, int32_t type, const regtopk_route_params* params, void* cuda_stream) {
  const size_t size = type_size(type);
  if (!size || tokens < 0 || n_experts < 1 || k < 1 || k > n_experts || !good_route(params, n_experts)) return REGTOPK_ERR_INVALID_ARG;
  if (n_experts > REGTOPK_ROUTE_MAX_EXPERTS || k > REGTOPK_ROUTE_MAX_CHOICES || params->groups > REGTOPK_ROUTE_MAX_GROUPS) return REGTOPK_ERR_TOO_LARGE;
  if (tokens == 0) return REGTOPK_OK;
  if (!good_matrix(logits, ld_logits, tokens, n_experts, size) || !good_matrix(experts, k, 1, k, 4) || !good_matrix(weights, k, 1, k, 4) ||
      (uintptr_t)bias % 4) return REGTOPK_ERR_INVALID_ARG;
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  RouteArgs a;
  a.logits = logits; a.bias = bias; a.experts = experts; a.weights = weights; a.ld = ld_logits; a.tokens = tokens; a.n_experts = n_experts; a.k = k;
  a.groups = params->groups; a.size = n_experts / params->groups; a.kept = params->groups_kept; a.top = params->group_top;
  a.lanes_log2 = 5;
  while (32 >> a.lanes_log2 < a.groups) --a.lanes_log2;
  a.lanes = 1 << a.lanes_log2;
  a.each = (a.size + a.lanes - 1) / a.lanes;
  a.sigmoid = params->scores == REGTOPK_SCORES_SIGMOID; a.renormalise = params->renormalise != 0; a.scale = params->scale;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  switch (type) {
    case REGTOPK_TYPE_F32: return launch_route_of<float>(a, sms, s);
    case REGTOPK_TYPE_BF16: return launch_route_of<__nv_bfloat16>(a, sms, s);
    default: return launch_route_of<__half>(a, sms, s);
  }
}

int regtopk_route_backward(const float* dweights, const void* logits, int64_t ld_logits, const int32_t* experts, void* dlogits,
                           int64_t ld_dlogits, int64_t tokens, int32_t n_experts, int32_t k, int32_t type,
                           const regtopk_route_params* params, void* cuda_stream) {
  const size_t size = type_size(type);
  if (!size || tokens < 0 || n_experts < 1 || k < 1 || k > n_experts || !good_route(params, n_experts)) return REGTOPK_ERR_INVALID_ARG;
  if (n_experts > REGTOPK_ROUTE_MAX_EXPERTS || k > REGTOPK_ROUTE_MAX_CHOICES || params->groups > REGTOPK_ROUTE_MAX_GROUPS) return REGTOPK_ERR_TOO_LARGE;
  if (tokens == 0) return REGTOPK_OK;
  if (!good_matrix(logits, ld_logits, tokens, n_experts, size) || !good_matrix(dlogits, ld_dlogits, tokens, n_experts, size) ||
      !good_matrix(experts, k, 1, k, 4) || !good_matrix(dweights, k, 1, k, 4)) return REGTOPK_ERR_INVALID_ARG;
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  RouteBackArgs a;
  a.dweights = dweights; a.logits = logits; a.experts = experts; a.dlogits = dlogits; a.ld = ld_logits; a.ldd = ld_dlogits; a.tokens = tokens;
  a.n_experts = n_experts; a.k = k; a.scale = params->scale;
  a.wide = n_experts % 8 == 0 && rows_aligned(logits, ld_logits, size, tokens) && rows_aligned(dlogits, ld_dlogits, size, tokens);
  a.sigmoid = params->scores == REGTOPK_SCORES_SIGMOID; a.renormalise = params->renormalise != 0;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  switch (type) {
    case REGTOPK_TYPE_F32: return launch_route_back<float>(a, sms, s);
    case REGTOPK_TYPE_BF16: return launch_route_back<__nv_bfloat16>(a, sms, s);
    default: return launch_route_back<__half>(a, sms, s);
  }
}

size_t regtopk_sort_tokens_workspace_bytes(int64_t tokens, int32_t k, int32_t n_experts, int32_t workers) {
  if (tokens < 0 || k < 1 || n_experts < 1 || workers < 1 || tokens > INT32_MAX / k || (int64_t)n_experts * workers > REGTOPK_MATMUL_MAX_GROUPS) return 0;
  const int64_t pairs = tokens * k, chunk = chunk_of(pairs), chunks = (pairs + chunk - 1) / chunk;
  return chunks <= 1 ? 0 : (size_t)chunks * n_experts * workers * sizeof(u32);
}

int regtopk_sort_tokens(const int32_t* experts, const int64_t* workers_at, int32_t workers, int64_t* offsets, int32_t* place,
                        int64_t tokens, int32_t k, int32_t n_experts, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (tokens < 0 || k < 1 || n_experts < 1 || workers < 1 || (!workers_at && workers != 1) || (uintptr_t)workers_at % 8 || !offsets ||
      (uintptr_t)offsets % 8) return REGTOPK_ERR_INVALID_ARG;
  if ((int64_t)n_experts * workers > REGTOPK_MATMUL_MAX_GROUPS || tokens > INT32_MAX / k) return REGTOPK_ERR_TOO_LARGE;
  if (tokens > 0 && (!good_matrix(experts, k, 1, k, 4) || !good_matrix(place, k, 1, k, 4))) return REGTOPK_ERR_INVALID_ARG;
  SortArgs a;
  a.experts = experts; a.workers_at = workers_at; a.offsets = offsets; a.place = place; a.tokens = tokens; a.pairs = tokens * k;
  a.k = divisor(k); a.workers = workers; a.n_experts = n_experts; a.groups = n_experts * workers;
  a.chunk = chunk_of(a.pairs);
  a.chunks = a.pairs ? (int)((a.pairs + a.chunk - 1) / a.chunk) : 1;
  a.counts = static_cast<u32*>(workspace);
  if (a.chunks > 1) {
    if (!workspace || (uintptr_t)workspace % 16) return REGTOPK_ERR_INVALID_ARG;
    if (workspace_bytes < regtopk_sort_tokens_workspace_bytes(tokens, k, n_experts, workers)) return REGTOPK_ERR_WORKSPACE_TOO_SMALL;
  }
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (a.chunks > 1) {
    const int rc = start(k_sort_count, a.chunks, kSortThreads, 0, s, a);
    if (rc != REGTOPK_OK) return rc;
  }
  constexpr int kMostSmem = REGTOPK_MATMUL_MAX_GROUPS * 4 * (1 + kSortWarps);
  if (!allow_smem_of<k_sort_place>(dev, kMostSmem)) return train_rc(cudaGetLastError());
  return start(k_sort_place, a.chunks, kSortThreads, (size_t)a.groups * 4 * (1 + kSortWarps), s, a);
}

}  // extern "C"
