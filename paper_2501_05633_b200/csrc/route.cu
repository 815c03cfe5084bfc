// The router: the choice of experts with its weights and their gradient, and the order of (worker, expert) groups
// (include/regtopk_experts.h).
//
// A token's logits are a few hundred numbers, so that a warp keeps them in registers and chooses by comparing there; the logits are
// read once.  What bounds the choice is the issue of instructions, not the memory: 32,768 tokens, eight of 256 experts by sigmoid scores with a
// bias in four of eight groups, take 36 to 39 us, 720 instructions of a warp a token, where 34 MB take 5.4 us; by bfloat16 logits alone 20 us.
// That is with numbers of which few are close.  Where equal ones are ordinary, tokens are worked out again in binary64, one after the other in their
// warp: bfloat16 logits with a bias of zeros 82 us, with one of multiples of 0.001 45 us, and where all logits are equal, as in a router that
// has not been trained, 215 to 228 us with a bias and 20 us without one.

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
  int places_log2, batch, share;  // places for a token's experts in a warp's lanes, at least k; tokens that a warp finishes together, and in all
  float scale;
};

// Binary32 numbers as whole numbers of the same order.  The number is canonical: no -0, and a NaN positive, as after an addition.
__device__ __forceinline__ u32 ordered(float v) {
  const u32 b = __float_as_uint(v);
  return b ^ ((u32)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(u32 o) { return __uint_as_float(o ^ ((u32)((int)~o >> 31) | 0x80000000u)); }
constexpr u32 kNone = 0x007FFFFFu;      // -infinity, with all low bits set: this and what is below is no expert
constexpr u32 kInfinite = 0xFF800000u;  // +infinity; NaN is above

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

// The weights of the experts chosen, one a lane and `places` lanes a token, as shares: exp(l) (softmax) or 1 / (1 + exp(-l)) over their
// sum.  Everything is taken relative to the largest, so that no sum is 0 whatever the logits.
__device__ __forceinline__ float share_of(float l, bool there, bool sigmoid, int places) {
  float most = there ? l : -INFINITY, v;
  for (int o = 1; o < places; o <<= 1) most = fmaxf(most, __shfl_xor_sync(kAll, most, o));
  if (sigmoid) {
    most = fminf(most, 0.0f);
    v = l < 0.0f ? expf(l - most) / (1.0f + expf(l)) : 1.0f / (1.0f + expf(-l));
  } else {
    v = expf(l - most);
  }
  if (!there) v = 0.0f;
  float total = v;
  for (int o = 1; o < places; o <<= 1) total += __shfl_xor_sync(kAll, total, o);
  return v / total;
}

// A token's weight of an expert with this logit; most, total: of all the token's logits, if not renormalised.
__device__ __forceinline__ float weight_of(const RouteArgs& a, float logit, bool there, int places, float most, float total) {
  if (a.renormalise) return share_of(logit, there, a.sigmoid, places);
  return a.sigmoid ? 1.0f / (1.0f + expf(-logit)) : expf(logit - most) / total;
}

// exp(x) for x <= 0 in binary64: x = n ln 2 + r (Cody and Waite, 1980), the exponential's series for |r| <= ln 2 / 2 to the thirteenth
// power, 2^-57 of it, and 2^n.  Without branches, so that those of a lane's experts overlap; below exp(-708) 0.
__device__ __forceinline__ double exp_64(double x) {
  const double n = rint(x * 1.4426950408889634), r = fma(n, -2.3190468138462996e-17, fma(n, -0.6931471805599453, x));
  double y = 1.0 / 6227020800.0;
  y = fma(y, r, 1.0 / 479001600.0);
  y = fma(y, r, 1.0 / 39916800.0);
  y = fma(y, r, 1.0 / 3628800.0);
  y = fma(y, r, 1.0 / 362880.0);
  y = fma(y, r, 1.0 / 40320.0);
  y = fma(y, r, 1.0 / 5040.0);
  y = fma(y, r, 1.0 / 720.0);
  y = fma(y, r, 1.0 / 120.0);
  y = fma(y, r, 1.0 / 24.0);
  y = fma(y, r, 1.0 / 6.0);
  y = fma(y, r, 0.5);
  y = fma(y, r, 1.0);
  y = fma(y, r, 1.0);
  y = y * __longlong_as_double((int64_t)(fmax(n, -1022.0) + 1023.0) << 52);
  return x < -708.0 ? 0.0 : y;  // a NaN stays one: r is
}
// 1 / x for 1 <= x <= 512 in binary64: binary32's, and Newton's method twice.
__device__ __forceinline__ double reciprocal_64(double x) {
  double y = reciprocal_fast((float)x);
  y = fma(y, fma(-x, y, 1.0), y);
  return fma(y, fma(-x, y, 1.0), y);
}

constexpr int kMostShare = 4096;  // tokens of a warp
// What a NaN counts as where groups are judged: below every binary32 number, and twice it is still above -infinity, which is a group
// that has no expert left.
constexpr double kNoNumber = -1e300;

// A token once more in binary64, for the few whose numbers lie too close for binary32.  slots and numbers: room for k and n_experts.
// The largest are looked for among the numbers rounded to binary32, which keeps their order; where several round to the same, the numbers
// themselves decide.
// What such a token costs is the time that a warp alone takes, binary64's operations above all.  So k_route leaves in the token's first
// expert the lanes whose groups remain, and in its first weight a number that the k largest reach: only what may reach it, in binary32, is
// worked out in binary64.  No lanes: it is not certain which groups remain, and everything is.
template <typename T, int N>
__device__ __noinline__ void route_in_64_bits(const RouteArgs& a, int64_t t, int* slots, double* numbers, int lane) {
  const T* row = static_cast<const T*>(a.logits) + t * a.ld;
  const Share own(a, lane);
  const u32 lanes = (u32)a.experts[t * a.k];
  const float reached = lanes ? a.weights[t * a.k] : -INFINITY;
  float l[N], most = -INFINITY;
  read_logits<T, N>(l, row, own, a.wide);
  bool bad = false;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    most = fmaxf(most, l[i]);
    bad |= !(l[i] <= FLT_MAX);
  }
  bad = __any_sync(kAll, bad);
  const bool judged = a.groups > 1 && a.top == 2, scored = a.bias || (judged && !lanes);
  double total = 1.0, per_total = 1.0;
  if (!a.sigmoid && (scored || !a.renormalise)) {
    most = warp_max(most);
    total = 0.0;
#pragma unroll 2
    for (int i = 0; i < own.count; ++i) total += exp_64((double)to_float(row[own.first + i]) - (double)most);
    total = warp_sum(total);
    per_total = reciprocal_64(total);
  }
  u32 todo = 0;  // of this lane's experts
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float c = l[i];
    if (a.bias) {
      const float s = a.sigmoid ? reciprocal_fast(1.0f + exp2_fast(c * -kLog2E)) : exp2_fast((c - most) * kLog2E) * (float)per_total;
      c = s + (i < own.count ? a.bias[own.first + i] : 0.0f);
    }
    if (l[i] != -INFINITY && !(c < reached) && (!lanes || (lanes >> lane & 1u))) todo |= 1u << i;
  }
  double t1 = -INFINITY, t2 = -INFINITY;  // of this lane, then of its group
  u32 key[N];
#pragma unroll
  for (int i = 0; i < N; ++i) key[i] = 0;
  for (; __any_sync(kAll, todo); todo &= todo - 1) {
    if (!todo) continue;
    const int at = __ffs(todo) - 1;
    const float logit = to_float(row[own.first + at]);
    double s = logit, c = logit;
    if (scored) {
      const double e = exp_64(a.sigmoid ? -fabs(s) : s - (double)most), r = a.sigmoid ? reciprocal_64(1.0 + e) : per_total;
      s = a.sigmoid && logit >= 0.0f ? r : e * r;
      if (a.bias) c = s = s + (double)a.bias[own.first + at];
    }
    numbers[own.first + at] = c;
    if (c == -INFINITY) s = -INFINITY;
    else if (s != s) s = kNoNumber;
    const u32 k = c == -INFINITY ? 0u : c != c ? 1u : ordered((float)c + 0.0f);
#pragma unroll
    for (int i = 0; i < N; ++i) key[i] = i == at ? k : key[i];
    t2 = fmax(t2, fmin(t1, s));
    t1 = fmax(t1, s);
  }
  const double* c = numbers + own.first;
  if (a.groups > 1 && !lanes) {
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
#pragma unroll
    for (int i = 0; i < N; ++i) key[i] = rank < a.kept ? key[i] : 0u;
  }
  int found = 0;
#pragma unroll 1
  for (; found < a.k; ++found) {
    u32 best = key[0];
#pragma unroll
    for (int i = 1; i < N; ++i) best = max(best, key[i]);
    const u32 m = __reduce_max_sync(kAll, best);
    if (m == 0) break;
    int at = -1;
    u32 open = 0;  // this lane's with that key, and the first of them
#pragma unroll
    for (int i = N - 1; i >= 0; --i) {
      open |= key[i] == m ? 1u << i : 0u;
      at = key[i] == m ? i : at;
    }
    u32 holders = __ballot_sync(kAll, at >= 0);
    if (m != 1u && __any_sync(kAll, (open & (open - 1)) || (holders & (holders - 1)))) {
      double largest = -INFINITY;
      if (at >= 0) {
#pragma unroll 1
        for (int i = 0; i < own.count; ++i)
          if (open >> i & 1u && c[i] > largest && ordered((float)c[i] + 0.0f) == m) {
            largest = c[i];
            at = i;
          }
      }
      double top = largest;
#pragma unroll
      for (int o = 16; o; o >>= 1) top = fmax(top, __shfl_xor_sync(kAll, top, o));
      holders = __ballot_sync(kAll, at >= 0 && largest == top);
    }
    if (lane == __ffs(holders) - 1) {
      slots[found] = own.first + at;
#pragma unroll
      for (int i = 0; i < N; ++i) key[i] = i == at ? 0u : key[i];
    }
  }
  __syncwarp();
  const bool there = lane < found;
  const int e = there ? slots[lane] : -1;
  __syncwarp();
  const float logit = there ? to_float(row[e]) : 0.0f;
  float w = weight_of(a, logit, there, 32, most, (float)total);
  if (bad && !a.sigmoid) w = __uint_as_float(0x7FC00000u);
  if (lane < a.k) {
    a.experts[t * a.k + lane] = e;
    a.weights[t * a.k + lane] = there ? w * a.scale : 0.0f;
  }
}

// Descending order within a lane, by the shortest networks for two, four and eight (Knuth, volume 3, 5.3.4).
__device__ __forceinline__ void exchange(u32& a, u32& b) {
  const u32 x = a;
  a = max(x, b);
  b = min(x, b);
}
template <int N> __device__ __forceinline__ void sort_descending(u32 (&v)[N]) {
  if constexpr (N == 2) {
    exchange(v[0], v[1]);
  } else if constexpr (N == 4) {
    exchange(v[0], v[2]); exchange(v[1], v[3]);
    exchange(v[0], v[1]); exchange(v[2], v[3]);
    exchange(v[1], v[2]);
  } else if constexpr (N == 8) {
    exchange(v[0], v[2]); exchange(v[1], v[3]); exchange(v[4], v[6]); exchange(v[5], v[7]);
    exchange(v[0], v[4]); exchange(v[1], v[5]); exchange(v[2], v[6]); exchange(v[3], v[7]);
    exchange(v[0], v[1]); exchange(v[2], v[3]); exchange(v[4], v[5]); exchange(v[6], v[7]);
    exchange(v[2], v[4]); exchange(v[3], v[5]);
    exchange(v[1], v[4]); exchange(v[3], v[6]);
    exchange(v[1], v[2]); exchange(v[3], v[4]); exchange(v[5], v[6]);
  }
}

template <int N> __device__ __forceinline__ u32 largest_of(const u32 (&v)[N]) {
  u32 m = v[0];
#pragma unroll
  for (int i = 1; i < N; ++i) m = max(m, v[i]);
  return m;
}
// The pair (x, y) to shared memory at `to` + `offset`, if a == y.
__device__ __forceinline__ void write_if(u32 a, u32 y, u32 to, int offset, int x) {
  asm volatile("{\n.reg .pred p;\nsetp.eq.u32 p, %0, %1;\n@p st.shared.v2.b32 [%2], {%3, %1};\n}" ::"r"(a), "r"(y), "r"(to + offset), "r"(x) : "memory");
}

// How experts are compared: by their logits (without bias: the order is the same), or by c, a score and its bias.  Judged: by their logits, but
// their groups by two scores.
enum How { kByLogit, kBySoftmax, kBySigmoid, kJudgedBySoftmax, kJudgedBySigmoid };

// A token's experts are found by k times taking the largest key of the warp.  A key is a number in the order of c whose low bits say
// which of the lane's experts it belongs to, so that one reduction finds number and place; a lane keeps its keys sorted.
//   16-bit logits that are compared themselves: the low bits of the numbers are 0, the expert's own number fits there, and the keys are in the exact
//   order, ties included.
//   Otherwise log2(N) bits are cut off and scores are rounded: tokens among whose first k + 1 numbers, or at the border of whose
//   groups, two are closer than both errors together are done again by route_in_64_bits, as are those with NaN.
// Errors, in units of 2^-24.  Sigmoid s: its argument x is rounded, which changes s by 0.224 * 1.25, the exponential is 2 units of its last
// place off, which changes s by 1, the sum is rounded, 1, and the reciprocal, 2: less than 8 for each, 2^-20 for a difference of two.
// Softmax: the exponential likewise (x exp(-x) is 0.37 at most), the sum of up to 512 of them, a tree of at most 21 additions, a reciprocal
// and a product: less than 2^-19 of the largest score, 2^-18 for a difference.
// The weights of a warp's `batch` tokens are worked out together, in lanes that would be idle with one token's (the
// first case above 47 us, one token at a time 57 us).  Four blocks an SM for up to eight experts a lane: with three, which need no spills,
// it takes 41 us, with five 47 us, where four take 39 us.
template <typename T, int N, int HOW>
__global__ void __launch_bounds__(kRouteThreads, N <= 8 ? 4 : 2) k_route(const __grid_constant__ RouteArgs a) {
  __shared__ int all_slots[kRouteWarps][32];
  __shared__ u32 all_unsure[kRouteWarps][kMostShare / 32];  // a bit for each of the warp's tokens
  __shared__ double all_numbers[kRouteWarps][REGTOPK_ROUTE_MAX_EXPERTS];
  __shared__ int2 all_found[kRouteWarps][64];  // of a token's keys: the holder's first expert, the key; and the key after the last
  begin_after_predecessor();
  constexpr bool kSorted = N <= 8;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, places = 1 << a.places_log2;
  int2* all = all_found[warp];
  u32* unsure = all_unsure[warp];
  const Share own(a, lane);
  constexpr bool kSigmoid = HOW == kBySigmoid || HOW == kJudgedBySigmoid, kSoftmax = HOW == kBySoftmax || HOW == kJudgedBySoftmax;
  constexpr bool by_logit = !(HOW == kBySoftmax || HOW == kBySigmoid), exact = sizeof(T) == 2 && by_logit;
  constexpr u32 low_bits = exact ? 511u : (u32)(N - 1);
  float bias[by_logit ? 1 : N];
  if (!by_logit) {
#pragma unroll
    for (int i = 0; i < N; ++i) bias[by_logit ? 0 : i] = i < own.count ? a.bias[own.first + i] : 0.0f;
  }
  int64_t t0 = ((int64_t)blockIdx.x * kRouteWarps + warp) * a.share;
  const int64_t end = min(t0 + a.share, a.tokens);
  const T* logits = static_cast<const T*>(a.logits);
  float ahead[N];
  if (t0 < end) read_logits<T, N>(ahead, logits + t0 * a.ld, own, a.wide);
  const int64_t begin = t0;
  for (int i = lane; i < (a.share + 31) >> 5; i += 32) unsure[i] = 0;
  bool any = false;
  __syncwarp();
  for (; t0 < end; t0 += a.batch) {
    int count = 0;           // this lane's token's: experts found,
    u32 lanes = kAll;        // lanes whose groups remain,
    float most = 0.0f, total = 1.0f, margin = 0.0f;  // largest logit, sum of the exponentials, error of a difference of scores
    u32 close = 0;           // a bit a token
    for (int r = 0; r < a.batch; ++r) {
      const int64_t t = t0 + r;
      if (t >= end) break;
      float l[N];
#pragma unroll
      for (int i = 0; i < N; ++i) l[i] = ahead[i];
      if (t + 1 < end) read_logits<T, N>(ahead, logits + (t + 1) * a.ld, own, a.wide);
      const bool mine = lane >> a.places_log2 == r;
      float top = 0.0f, sum = 1.0f, per_sum = 1.0f;
      if (kSoftmax || (!kSigmoid && !a.sigmoid && !a.renormalise)) {
        top = l[0];
#pragma unroll
        for (int i = 1; i < N; ++i) top = fmaxf(top, l[i]);
        top = warp_max(top);
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) sum += exp2_fast((l[i] == -INFINITY ? -INFINITY : l[i] - top) * kLog2E);
        sum = warp_sum(sum);
        per_sum = 1.0f / sum;
        if (mine) most = top, total = sum;
      }
      const float apart = HOW == kByLogit ? 0.0f : kSigmoid ? 0x1p-20f : 0x1p-18f * per_sum;
      if (mine) margin = apart;
      u32 key[N];
      float t1 = -INFINITY, t2 = -INFINITY;  // the two largest scores, of this lane and then of its group
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float c = l[i];
        const u32 low = exact ? 511u - (u32)(own.first + i) & 511u : (u32)(N - 1 - i);  // behind the last expert it may wrap
        if (HOW != kByLogit) {
          const float s = kSigmoid ? reciprocal_fast(1.0f + exp2_fast(c * -kLog2E)) : exp2_fast((c - top) * kLog2E) * per_sum;
          const float scored = c == -INFINITY ? -INFINITY : by_logit ? s : s + bias[by_logit ? 0 : i];
          t2 = fmaxf(t2, fminf(t1, scored));
          t1 = fmaxf(t1, scored);
          if (!by_logit) c = scored;
        }
        if (by_logit) c += 0.0f;
        key[i] = (ordered(c) & ~low_bits) | low;
      }
      if (kSorted) sort_descending<N>(key);
      bool near = false;
      if (a.groups > 1) {
        u32 group, last = 0, next = 0;
        bool kept = false;
        if (HOW == kByLogit) {
          // judged by the largest logit: its key, of which the low bits may be the group's
          u32 best = kSorted ? key[0] : largest_of<N>(key);
          for (int o = 1; o < a.lanes; o <<= 1) best = max(best, __shfl_xor_sync(kAll, best, o));
          group = own.group < a.groups ? (best & ~(exact ? 511u : 31u)) | (31u - own.group) : 0u;
        } else {
          for (int o = 1; o < a.lanes; o <<= 1) {
            const float o1 = __shfl_xor_sync(kAll, t1, o), o2 = __shfl_xor_sync(kAll, t2, o);
            t2 = fmaxf(fminf(t1, o1), fmaxf(t2, o2));
            t1 = fmaxf(t1, o1);
          }
          const float strength = (a.top == 2 && t2 > -INFINITY ? t1 + t2 : t1) + 0.0f;
          group = own.group < a.groups ? ordered(strength) : 0u;
        }
        for (int g = 0; g < a.kept; ++g) {
          last = __reduce_max_sync(kAll, group);
          kept |= group == last;
          group = group == last ? 0u : group;
        }
        next = __reduce_max_sync(kAll, group);
        u32 those = __ballot_sync(kAll, kept);
        if (HOW == kByLogit) {
          const float v = unordered(last & ~31u), w = unordered(next & ~31u);
          near = !exact && a.kept < a.groups && w > -INFINITY && !(v - w > 0x1p-17f * (fabsf(v) + fabsf(w)));
        } else {
          // more groups than there may be, because two are of one strength; a NaN, which the maxima pass over; or a border that is too close
          const float size = own.group < a.groups && t1 > -INFINITY ? fabsf(t1) + (a.top == 2 && t2 > -INFINITY ? fabsf(t2) : 0.0f) : 0.0f;  // two scores may cancel
          const float most_size = __uint_as_float(__reduce_max_sync(kAll, __float_as_uint(size)));
          const float v = unordered(last), w = a.kept < a.groups ? unordered(next) : -INFINITY;
          near = __popc(those & __ballot_sync(kAll, t1 > -INFINITY)) > a.kept << a.lanes_log2 || (w > -INFINITY && !(v - w > fmaf(0x1p-22f, most_size, 2.0f * apart)));
          near |= __any_sync(kAll, (kSorted ? key[0] : largest_of<N>(key)) > (kInfinite | low_bits));
          if (HOW == kJudgedBySoftmax) near |= sum != sum;  // +infinity among the logits: no key is NaN, but every score
        }
#pragma unroll
        for (int i = 0; i < N; ++i) key[i] = kept ? key[i] : 0u;
        those = near ? 0u : those;
        if (mine) lanes = those;
      }
      // the k largest keys and the one after them, four at a time.  The lane that holds one writes it down and goes on to its next; without
      // branches, which would take longer than all this.  What is no expert is written down too.
      int found = 0, taken = 0;
      const u32 slot = smem_at(all) + r * (places + 1) * 8;
      for (int j0 = 0; j0 <= a.k; j0 += 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (j > 0 && j0 + j > a.k) break;
          u32 best = kSorted ? key[0] : largest_of<N>(key);
          const u32 m = __reduce_max_sync(kAll, best);
          const bool holds = best == m, real = m > kNone;
          write_if(best, m, slot + j0 * 8, j * 8, own.first);
          found += real;
          taken += holds && real;
          if (kSorted) {
#pragma unroll
            for (int i = 0; i + 1 < N; ++i) key[i] = holds ? key[i + 1] : key[i];
            key[N - 1] = holds ? 0u : key[N - 1];
          } else {
#pragma unroll
            for (int i = 0; i < N; ++i) key[i] = key[i] == m ? 0u : key[i];
          }
        }
      }
      if (!exact) near |= __reduce_add_sync(kAll, taken) != found;  // the same key twice
      if (near) close |= 1u << r;
      if (mine) count = min(found, a.k);
    }
    __syncwarp();
    // from here on a lane has one place of one token
    const int r = lane >> a.places_log2, j = lane & (places - 1);
    const int64_t t = t0 + r;
    u32 first = 0;
    bool near = false;
    int e = -1;
    if (count > 0) {
      const int2* slot = all + r * (places + 1);
      first = (u32)slot[0].y;
      if (j < count) {
        const u32 k = (u32)slot[j].y, next = (u32)slot[j + 1].y;
        const float v = unordered(k & ~low_bits), w = unordered(next & ~low_bits);
        near = k > (kInfinite | low_bits) || (!exact && next > kNone && !(v - w > fmaf(N * 0x1p-22f, fabsf(v) + fabsf(w), by_logit ? 0.0f : margin)));
        e = exact ? (int)(511u - (k & 511u)) : slot[j].x + N - 1 - (int)(k & (N - 1));
      }
    }
    near |= (close >> r & 1u) != 0;
    const u32 all_near = __ballot_sync(kAll, near);
    if (all_near) {
      any = true;
      if (near && t < end) atomicOr(&unsure[(t - begin) >> 5], 1u << ((t - begin) & 31));
      if (all_near >> (r << a.places_log2) & (0xFFFFFFFFu >> (32 - places))) near = true;
    }
    const bool there = j < count;
    const float logit = there ? to_float(logits[t * a.ld + e]) : 0.0f;
    float w = weight_of(a, logit, there, places, most, total);
    // a NaN or an infinity anywhere makes the scores of a softmax NaN
    if (!a.sigmoid && (kSoftmax ? total != total : first >= kInfinite)) w = __uint_as_float(0x7FC00000u);
    if (j < a.k && r < a.batch && t < end) {
      w = there ? w * a.scale : 0.0f;
      if (near && j == 0) {  // what route_in_64_bits goes on from
        const bool strange = first > (kInfinite | low_bits);  // a NaN, which came first here and comes last there
        e = strange ? 0 : (int)lanes;
        w = -INFINITY;
        if (count == a.k && !strange) {
          const float v = unordered((u32)all[r * (places + 1) + a.k - 1].y & ~low_bits);
          w = v - fmaf(N * 0x1p-21f, fabsf(v), 2.0f * margin);
          if (!(w == w)) w = -INFINITY;
        }
      }
      a.experts[t * a.k + j] = e;
      a.weights[t * a.k + j] = w;
    }
    __syncwarp();
  }
  if (!any) return;
  for (int64_t t = begin; t < end; ++t)
    if (unsure[(t - begin) >> 5] >> ((t - begin) & 31) & 1u) route_in_64_bits<T, N>(a, t, all_slots[warp], all_numbers[warp], lane);
}

// ---- the gradient to the logits ------------------------------------------------------------------------------------
struct RouteBackArgs {
  const float* dweights;
  const void* logits;
  const int32_t* experts;
  void* dlogits;
  int64_t ld, ldd, tokens;
  int n_experts, k, wide, sigmoid, renormalise;
  int pitch, places_log2, batch;  // pitch: of a token's row in shared memory, odd
  Divisor columns;
  float scale;
};

// A warp takes `batch` tokens at a time, a token's chosen experts in `places` of its lanes.  What reaches their scores, or logits, is laid
// into rows in shared memory, from which the gradient's rows are written.  Plain softmax scores need all logits, the others only the
// chosen ones.  Latency bounds it.  For many tokens over up to 64 experts: 16,384 over eight take 5.1 us, with a token a warp 10.8 us; over
// 64, 7 us and 10 us; but over 256, 12.3 us and 9.7 us.  A quarter as many where all logits are needed, of which few lanes sum up a
// token's: 5,003 tokens over 60 take 8.5 us, with a token a warp 5 us.
constexpr int kBackRoom = 544, kBackMost = 64;  // numbers: several rows; the most experts
template <typename T> __global__ void __launch_bounds__(kRouteThreads) k_route_back(const __grid_constant__ RouteBackArgs a) {
  __shared__ float all_logits[kRouteWarps][kBackRoom], all_rows[kRouteWarps][kBackRoom];
  begin_after_predecessor();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, places = 1 << a.places_log2, r = lane >> a.places_log2, j = lane & (places - 1);
  float *logits = all_logits[warp], *rows = all_rows[warp];
  const float *own_logits = logits + r * a.pitch;
  const bool dense = !a.sigmoid && !a.renormalise;
  const auto sum = [&](float v) {
    for (int o = 1; o < places; o <<= 1) v += __shfl_xor_sync(kAll, v, o);
    return v;
  };
  const int64_t step = (int64_t)gridDim.x * kRouteWarps * a.batch;
  for (int64_t t0 = ((int64_t)blockIdx.x * kRouteWarps + warp) * a.batch; t0 < a.tokens; t0 += step) {
    const int count = (int)min((int64_t)a.batch, a.tokens - t0), all = count * a.n_experts;
    const T* from = static_cast<const T*>(a.logits) + t0 * a.ld;
    T* out = static_cast<T*>(a.dlogits) + t0 * a.ldd;
    const bool used = r < count && j < a.k;
    const int e = used ? a.experts[(t0 + r) * a.k + j] : -1;
    const bool there = e >= 0 && e < a.n_experts;
    const float dw = there ? a.dweights[(t0 + r) * a.k + j] : 0.0f, l = there ? to_float(from[r * a.ld + e]) : 0.0f;
#pragma unroll 4
    for (int n = lane; n < all; n += 32) {
      const int row = (int)a.columns.quotient_of((u32)n), i = n - row * a.n_experts;
      rows[row * a.pitch + i] = 0.0f;
      if (dense) logits[row * a.pitch + i] = to_float(from[row * a.ld + i]);
    }
    __syncwarp();
    float most = -INFINITY, per_total = 0.0f, mean = 0.0f, g;
    if (dense) {
      if (r < count)
        for (int i = j; i < a.n_experts; i += places) most = fmaxf(most, own_logits[i]);
      for (int o = 1; o < places; o <<= 1) most = fmaxf(most, __shfl_xor_sync(kAll, most, o));
      float total = 0.0f;
      if (r < count)
        for (int i = j; i < a.n_experts; i += places) total += own_logits[i] == -INFINITY ? 0.0f : expf(own_logits[i] - most);
      total = sum(total);
      per_total = total > 0.0f ? 1.0f / total : total;  // a row without experts has no scores
      g = a.scale * dw;
      mean = sum(there && l != -INFINITY ? g * expf(l - most) * per_total : 0.0f);
    } else if (a.renormalise) {
      const float p = share_of(l, there, a.sigmoid, places);
      g = a.scale * p * (dw - sum(there ? dw * p : 0.0f));
      if (a.sigmoid) g /= 1.0f + expf(l);
    } else {
      const float q = expf(-fabsf(l)), s = 1.0f / (1.0f + q);
      g = a.scale * dw * (q * s) * s;
    }
    float* target = rows + r * a.pitch + (there ? e : 0);
    const u32 same = __match_any_sync(kAll, there ? r * a.pitch + e : -1 - lane);
    if (__any_sync(kAll, there && (same & (same - 1)))) {  // the same expert twice: one after the other, in order
      for (int i = 0; i < a.k; ++i) {
        if (j == i && there) *target += g;
        __syncwarp();
      }
    } else if (there) {
      *target = g;
    }
    __syncwarp();
#pragma unroll 4
    for (int n0 = 0; n0 < all; n0 += 32) {
      const int n = min(n0 + lane, all - 1), row = (int)a.columns.quotient_of((u32)n), i = n - row * a.n_experts;
      float f = rows[row * a.pitch + i];
      if (dense) {
        const int first = row << a.places_log2;
        const float x = logits[row * a.pitch + i], top = __shfl_sync(kAll, most, first), per = __shfl_sync(kAll, per_total, first), m = __shfl_sync(kAll, mean, first);
        f = x == -INFINITY ? 0.0f : expf(x - top) * per * (f - m);
      }
      if (n0 + lane < all) out[row * a.ldd + i] = from_float<T>(f);
    }
    __syncwarp();
  }
}

// A warp a token, for more experts.
template <typename T> __global__ void __launch_bounds__(kRouteThreads) k_route_back_row(const __grid_constant__ RouteBackArgs a) {
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
      const float p = share_of(l, there, a.sigmoid, 32);
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
// warp.  Where a pair goes: to the start of its group, past the pairs of the group in the chunks before, in the runs before and in its own
// run, which a warp goes through in steps of 32.  Nothing depends on the order in which blocks or warps run.
//   Up to 4,096 pairs: one block.  Up to 16,384: a cluster of eight, which read one another's counts in shared memory.  More: k_sort_count
//   counts the chunks first, and every block adds up the counts of all of them, 128 at most.  Above 1 million pairs k_sort_scan adds them up once for
//   all blocks, because that sum would grow with the square of the pairs (2^31 of them: 65,536 blocks, 65,536 chunks each): 4 million pairs in
//   256 groups take 84 us (147 us with a sum in every block), 134 million 2.3 ms.
// It is latency that these take: two reads from memory one after the other (experts, and workers beside them), barriers, one write.  3,000
// pairs 6 us, 65,536 pairs in two launches 7 us over 8 groups and 10 us over 256 (with cold caches 12.5 us, and a cluster of eight with 8,192 pairs a
// block 14.6 us, most of it for comparing the groups of 32 neighbours).
struct SortArgs {
  const int32_t* experts;
  const int64_t* workers_at;  // NULL: all tokens are of worker 0
  int64_t* offsets;
  int32_t* place;
  u32* counts;  // [chunks][groups]; of long sorts what lies in the chunks before, and [chunks]: the groups' sizes
  int64_t tokens, pairs;
  Divisor k;
  int workers, n_experts, groups, chunk, chunks;
};

constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kSortKept = 8;  // steps of a run whose groups stay in registers between the two times that they are needed
constexpr int kSortCluster = 8;

// The group of a pair, or -1; `at` is a copy of workers_at in shared memory.
__device__ __forceinline__ int group_of_pair(const SortArgs& a, const int64_t* at, u32 pair, int e) {
  if (e < 0 || e >= a.n_experts) return -1;
  if (!a.workers_at) return e;
  const int64_t t = a.k.quotient_of(pair);
  if (t < at[0] || t >= at[a.workers]) return -1;
  int lo = 0, hi = a.workers;  // the last worker that begins at t or before
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (at[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo * a.n_experts + e;
}
__device__ __forceinline__ void copy_workers(const SortArgs& a, int64_t* at) {
  if (a.workers_at)
    for (int i = threadIdx.x; i <= a.workers; i += kSortThreads) at[i] = a.workers_at[i];
}

__global__ void __launch_bounds__(kSortThreads) k_sort_count(const __grid_constant__ SortArgs a) {
  __shared__ u32 count[REGTOPK_MATMUL_MAX_GROUPS];
  __shared__ int64_t workers_at[REGTOPK_MATMUL_MAX_GROUPS + 1];
  begin_after_predecessor();
  copy_workers(a, workers_at);
  for (int g = threadIdx.x; g < a.groups; g += kSortThreads) count[g] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * a.chunk, end = min(first + a.chunk, a.pairs);
  for (int64_t p = first + threadIdx.x; p < end; p += kSortThreads) {
    const int g = group_of_pair(a, workers_at, (u32)p, a.experts[p]);
    if (g >= 0) atomicAdd(&count[g], 1u);
  }
  __syncthreads();
  for (int g = threadIdx.x; g < a.groups; g += kSortThreads) a.counts[(int64_t)blockIdx.x * a.groups + g] = count[g];
}

// The counts of every chunk become the sums over the chunks before it, and the groups' sizes follow the last.  A block has 32 groups, which
// are neighbours in memory, and a warp one of 32 runs of chunks.
__global__ void __launch_bounds__(kSortThreads) k_sort_scan(const __grid_constant__ SortArgs a) {
  __shared__ u32 sums[kSortWarps][32];
  begin_after_predecessor();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = blockIdx.x * 32 + lane;
  const int length = (a.chunks + kSortWarps - 1) / kSortWarps, first = min(warp * length, a.chunks), end = min(first + length, a.chunks);
  u32 sum = 0;
  if (g < a.groups) {
#pragma unroll 8
    for (int c = first; c < end; ++c) sum += a.counts[(int64_t)c * a.groups + g];
  }
  sums[warp][lane] = sum;
  __syncthreads();
  u32 before = 0;
  for (int w = 0; w < warp; ++w) before += sums[w][lane];
  if (g >= a.groups) return;
#pragma unroll 8
  for (int c = first; c < end; ++c) {
    u32* at = a.counts + (int64_t)c * a.groups + g;
    const u32 n = *at;
    *at = before;
    before += n;
  }
  if (warp == kSortWarps - 1) a.counts[(int64_t)a.chunks * a.groups + g] = before;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ u32 load_of_block(const u32* own, u32 block) {  // what lies at this place in another block's shared memory
  u32 at, v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_at(own)), "r"(block));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at));
  return v;
}

// How the chunks of a sort know of one another.
enum Chunks { kOneBlock, kOneCluster, kCountedBefore, kCountedLong };  // kCountedLong: runs of more than kSortKept steps, counts that are sums

// dynamic shared memory: workers_at; of each group its size and what lies before it [2][groups], then runs [warps][groups]
template <int CHUNKS> __global__ void __launch_bounds__(kSortThreads) k_sort_place(const __grid_constant__ SortArgs a) {
  extern __shared__ __align__(16) char smem[];
  __shared__ u32 sums[kSortWarps];
  typedef uint16_t Run;  // a chunk has at most 32,768 pairs
  constexpr bool kKept = CHUNKS != kCountedLong;
  begin_after_predecessor();
  int64_t* workers_at = reinterpret_cast<int64_t*>(smem);
  u32 *base = reinterpret_cast<u32*>(workers_at + a.workers + 1), *sizes = base + a.groups;
  Run* runs = reinterpret_cast<Run*>(sizes + a.groups);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // this warp's run
  const int64_t first = (int64_t)blockIdx.x * a.chunk, end = min(first + a.chunk, a.pairs), pairs = max(end - first, (int64_t)0);
  const int64_t length = ((pairs + kSortWarps - 1) / kSortWarps + 31) & ~31ll, from = first + warp * length, to = min(from + length, end);
  int kept[kKept ? kSortKept : 1];
  if (kKept) {
#pragma unroll
    for (int i = 0; i < kSortKept; ++i) kept[i] = from + i * 32 + lane < to ? a.experts[from + i * 32 + lane] : -1;
  }
  copy_workers(a, workers_at);
  for (int i = threadIdx.x; i < 2 * a.groups; i += kSortThreads) base[i] = 0;
  for (int i = threadIdx.x; i < kSortWarps * a.groups; i += kSortThreads) runs[i] = 0;
  __syncthreads();
  Run* own = runs + warp * a.groups;
#pragma unroll kKept ? kSortKept : 1
  for (int i = 0; kKept ? i < kSortKept : from + i * 32 < to; ++i) {
    if (kKept && from + i * 32 >= to) break;
    const int64_t p = from + i * 32 + lane;
    const int g = p < to ? group_of_pair(a, workers_at, (u32)p, kKept ? kept[kKept ? i : 0] : a.experts[p]) : -1;
    if (kKept) kept[kKept ? i : 0] = g;
    const u32 same = __match_any_sync(kAll, g);
    if (g >= 0 && lane == __ffs(same) - 1) own[g] += (Run)__popc(same);
    __syncwarp();
  }
  // the sums over chunks that have been counted before, by as many threads a group as there are
  if (CHUNKS == kCountedLong) {
    for (int g = threadIdx.x; g < a.groups; g += kSortThreads) {
      sizes[g] = a.counts[(int64_t)a.chunks * a.groups + g];
      base[g] = a.counts[(int64_t)blockIdx.x * a.groups + g];
    }
  }
  if (CHUNKS == kCountedBefore) {
    const int parts = a.groups >= kSortThreads ? 1 : kSortThreads / a.groups;
    for (int i = threadIdx.x; i < parts * a.groups; i += kSortThreads) {
      const int part = i / a.groups, g = i - part * a.groups;
      u32 total = 0, before = 0;
#pragma unroll 8
      for (int c = part; c < a.chunks; c += parts) {
        const u32 n = a.counts[(int64_t)c * a.groups + g];
        total += n;
        before += c < (int)blockIdx.x ? n : 0;
      }
      atomicAdd(&sizes[g], total);
      atomicAdd(&base[g], before);
    }
  }
  __syncthreads();
  // what lies in the runs before, and the size of the chunk's share
  for (int g = threadIdx.x; g < a.groups; g += kSortThreads) {
    u32 here = 0;
#pragma unroll 8
    for (int w = 0; w < kSortWarps; ++w) {
      const u32 n = runs[w * a.groups + g];
      runs[w * a.groups + g] = (Run)here;
      here += n;
    }
    if (CHUNKS == kOneBlock || CHUNKS == kOneCluster) sizes[g] = here;
  }
  if (CHUNKS == kOneCluster) {
    cluster_arrive();
    cluster_wait();
  }
  // of every group: its size, and what lies in the groups and chunks before
  u32 at = 0;  // start of the groups that this round of threads looks at
  for (int g0 = 0; g0 < a.groups; g0 += kSortThreads) {
    const int g = g0 + threadIdx.x;
    u32 total = 0, before = 0;
    if (g < a.groups) {
      if (CHUNKS == kOneCluster) {
        u32 n[kSortCluster];
#pragma unroll
        for (u32 c = 0; c < kSortCluster; ++c) n[c] = load_of_block(&sizes[g], c);
#pragma unroll
        for (u32 c = 0; c < kSortCluster; ++c) {
          total += n[c];
          before += c < blockIdx.x ? n[c] : 0;
        }
      } else {
        total = sizes[g];
        before = base[g];
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
    u32 before_warps = sums[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u32 v = __shfl_up_sync(kAll, before_warps, o);
      if (lane >= o) before_warps += v;
    }
    const u32 all = __shfl_sync(kAll, before_warps, 31), lower = at + (warp ? __shfl_sync(kAll, before_warps, warp - 1) : 0);
    if (g < a.groups) {
      base[g] = lower + scan - total + before;
      if (blockIdx.x == 0) {
        a.offsets[g] = lower + scan - total;
        if (g == a.groups - 1) a.offsets[a.groups] = lower + scan;
      }
    }
    at += all;
    __syncthreads();
  }
  if (CHUNKS == kOneCluster) cluster_arrive();  // the others' counts have been read
#pragma unroll kKept ? kSortKept : 1
  for (int i = 0; kKept ? i < kSortKept : from + i * 32 < to; ++i) {
    if (kKept && from + i * 32 >= to) break;
    const int64_t p = from + i * 32 + lane;
    const int g = kKept ? kept[kKept ? i : 0] : p < to ? group_of_pair(a, workers_at, (u32)p, a.experts[p]) : -1;
    const u32 same = __match_any_sync(kAll, g);
    const u32 rank = __popc(same & ((1u << lane) - 1));
    u32 where = 0;
    if (g >= 0) where = base[g] + own[g] + rank;
    __syncwarp();
    if (g >= 0 && rank == 0) own[g] += (Run)__popc(same);
    __syncwarp();
    if (p < to) a.place[p] = g >= 0 ? (int32_t)where : -1;
  }
  if (CHUNKS == kOneCluster) cluster_wait();  // and this one's, before its shared memory is another's
}

// Pairs of a chunk.
constexpr int64_t kMostOfBlock = 4096, kMostOfCluster = (int64_t)kSortCluster * 2 * kSortThreads, kMostKept = kSortKept * kSortThreads;
inline int chunk_of(int64_t pairs) {
  if (pairs <= kMostOfBlock) return (int)kMostOfBlock;
  if (pairs <= kMostOfCluster) return (int)((pairs + kSortCluster - 1) / kSortCluster);
  int64_t chunk = 1024;
  while (chunk * 128 < pairs && chunk < 32768) chunk *= 2;
  return (int)chunk;
}

constexpr size_t sort_smem(size_t groups, size_t workers) { return groups * (8 + kSortWarps * sizeof(uint16_t)) + 8 * (workers + 1); }

template <auto kKernel> bool allow_smem_of(int dev, int bytes) {
  static uint64_t done;  // of this kernel, one bit a device
  if (__atomic_load_n(&done, __ATOMIC_RELAXED) >> dev & 1) return true;
  if (cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
  __atomic_fetch_or(&done, 1ull << dev, __ATOMIC_RELAXED);
  return true;
}

template <typename T, int N> int launch_route(RouteArgs& a, int sms, cudaStream_t s) {
  // Every warp takes the same number of tokens, neighbours.  Finished together are as many as have places in a warp.
  a.places_log2 = 0;
  while (1 << a.places_log2 < a.k) ++a.places_log2;
  const int64_t warps = (int64_t)sms * (N <= 8 ? 4 : 2) * kRouteWarps;
  int64_t each = (a.tokens + warps - 1) / warps;
  if (each > kMostShare) each = kMostShare;
  if (a.tokens / each / kRouteWarps >= INT32_MAX) return REGTOPK_ERR_TOO_LARGE;
  a.share = (int)each;
  a.batch = 1;
  while (a.batch << a.places_log2 < 32 && a.batch < 8 && a.batch < each) a.batch *= 2;
  const unsigned grid = (unsigned)((a.tokens + each * kRouteWarps - 1) / (each * kRouteWarps));
  if (a.bias)
    return a.sigmoid ? start(k_route<T, N, kBySigmoid>, grid, kRouteThreads, 0, s, a) : start(k_route<T, N, kBySoftmax>, grid, kRouteThreads, 0, s, a);
  if (a.groups > 1 && a.top == 2)
    return a.sigmoid ? start(k_route<T, N, kJudgedBySigmoid>, grid, kRouteThreads, 0, s, a) : start(k_route<T, N, kJudgedBySoftmax>, grid, kRouteThreads, 0, s, a);
  return start(k_route<T, N, kByLogit>, grid, kRouteThreads, 0, s, a);
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
template <typename T> int launch_route_back(RouteBackArgs& a, int sms, cudaStream_t s) {
  a.columns = divisor(a.n_experts);
  a.pitch = a.n_experts | 1;
  a.places_log2 = 0;
  while (1 << a.places_log2 < a.k) ++a.places_log2;
  a.batch = 1;  // as many as have places and room, while every SM has sixteen warps' work
  while (a.batch << a.places_log2 < 32 && 2 * a.batch * a.pitch <= kBackRoom && a.tokens >= (int64_t)sms * 16 * 2 * a.batch) a.batch *= 2;
  if (a.batch == 1 || a.n_experts > (a.sigmoid || a.renormalise ? kBackMost : kBackMost / 4)) {
    const int64_t blocks = (a.tokens + kRouteWarps - 1) / kRouteWarps, most = (int64_t)sms * 8;
    return start(k_route_back_row<T>, (unsigned)(blocks < most ? blocks : most), kRouteThreads, 0, s, a);
  }
  const int64_t each = kRouteWarps * a.batch, blocks = (a.tokens + each - 1) / each, most = (int64_t)sms * 6;
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
  const int64_t pairs = tokens * k, chunk = chunk_of(pairs);
  return pairs <= kMostOfCluster ? 0 : (size_t)((pairs + chunk - 1) / chunk + (chunk > kMostKept)) * n_experts * workers * sizeof(u32);
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
  const bool counted = a.pairs > kMostOfCluster;
  if (counted) {
    if (!workspace || (uintptr_t)workspace % 16) return REGTOPK_ERR_INVALID_ARG;
    if (workspace_bytes < regtopk_sort_tokens_workspace_bytes(tokens, k, n_experts, workers)) return REGTOPK_ERR_WORKSPACE_TOO_SMALL;
  }
  int dev, sms;
  if (!current_device(&dev, &sms)) return REGTOPK_ERR_NO_DEVICE;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const bool is_long = a.chunk > kMostKept;
  const size_t bytes = sort_smem(a.groups, workers), most = sort_smem(REGTOPK_MATMUL_MAX_GROUPS, REGTOPK_MATMUL_MAX_GROUPS);
  if (!counted) {
    if (a.pairs > kMostOfBlock) {
      if (!allow_smem_of<k_sort_place<kOneCluster>>(dev, (int)most)) return train_rc(cudaGetLastError());
      return start<kSortCluster>(k_sort_place<kOneCluster>, kSortCluster, kSortThreads, bytes, s, a);
    }
    if (!allow_smem_of<k_sort_place<kOneBlock>>(dev, (int)most)) return train_rc(cudaGetLastError());
    return start(k_sort_place<kOneBlock>, 1, kSortThreads, bytes, s, a);
  }
  const int rc = start(k_sort_count, a.chunks, kSortThreads, 0, s, a);
  if (rc != REGTOPK_OK) return rc;
  if (!is_long) {
    if (!allow_smem_of<k_sort_place<kCountedBefore>>(dev, (int)most)) return train_rc(cudaGetLastError());
    return start(k_sort_place<kCountedBefore>, a.chunks, kSortThreads, bytes, s, a);
  }
  if (!allow_smem_of<k_sort_place<kCountedLong>>(dev, (int)most)) return train_rc(cudaGetLastError());
  const int scanned = start(k_sort_scan, (a.groups + 31) / 32, kSortThreads, 0, s, a);
  if (scanned != REGTOPK_OK) return scanned;
  return start(k_sort_place<kCountedLong>, a.chunks, kSortThreads, bytes, s, a);
}

}  // extern "C"
