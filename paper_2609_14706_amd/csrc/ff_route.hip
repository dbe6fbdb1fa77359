// Routing to experts: from each token's logits to the experts that it takes, their
// weights, and the slots (token, choice) sorted by expert; the weights' gradient.
//
//   s_e = softmax_e(l) or sigmoid(l_e);  c_e = s_e + bias_e
//   groups of experts: the top_groups whose two best c sum to most are kept
//   chosen: the `top` largest c, the lowest index among equals
//   w_j = scale s_j, or scale s_j / sum of the chosen s
//
// Scores are held in 64 bits: which expert is chosen may hang on the last bit of c,
// and 32 bits of exp would decide otherwise than the formula for about one token in
// ten thousand.  A row of 16 lanes takes a token (for many experts or choices a whole wave),
// V neighbouring experts a lane; it picks one expert after the other, each the largest of
// the lanes' best: c as a whole number that orders alike, its high words compared first
// across the lanes (DPP), the low ones only where two lanes share the high one.  What
// bounds it is instructions, 2200 a token by whole waves: 16384 tokens, 8 of 256 experts in
// 8 groups, 36 us so and 26 by rows, the sort's two launches 5 each (their bytes: 4 us in all).
// One token's 8 of 128: 7.4 us, the latency of the steps one after the other.
//
// The sort is a counting sort, stable and without an atomic on memory: chunks of
// tokens count their slots by expert (k_route), a wave for each expert sums the chunks'
// counts (k_scan), and each chunk places its own slots (k_place): a wave takes 64 at a time,
// a slot's rank among those of its expert by ballots over the expert's bits.  Few
// tokens do all of it in one workgroup and one launch.
#include <math.h>

#include <algorithm>

#include "ff_common.hpp"
#include "ff_expert_kernels.hpp"
#include "ff_vec.hpp"

namespace ff {
namespace {

typedef unsigned long long u64;

// Largest 32-bit value of the wave, in every lane.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t from_lane(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, true);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max(v, from_lane<0x111, 0xf>(v));  // row_shr 1, 2, 4, 8: lane 15 of a row holds its largest
  v = max(v, from_lane<0x112, 0xf>(v));
  v = max(v, from_lane<0x114, 0xf>(v));
  v = max(v, from_lane<0x118, 0xf>(v));
  v = max(v, from_lane<0x142, 0xa>(v));  // row_bcast 15, 31: lane 63 the wave's
  v = max(v, from_lane<0x143, 0xc>(v));
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// A whole number that orders as c does, above 0 (which is "not to be chosen"); a
// NaN counts as the lowest value.
__device__ __forceinline__ u64 key_of(double c) {
  if (c != c) c = -INFINITY;
  const u64 b = (u64)__double_as_longlong(c);
  return b >> 63 ? ~b : b | 0x8000000000000000ull;
}

// The lane that holds the largest of the lanes' keys, the lowest one among equals
// (lanes hold ascending experts).
__device__ __forceinline__ int best_lane(u64 mine) {
  const uint32_t hi = (uint32_t)(mine >> 32), top = wave_max(hi);
  u64 who = __ballot(hi == top);
  if (who & (who - 1)) {
    const uint32_t lo = hi == top ? (uint32_t)mine : 0u, low = wave_max(lo);
    who = __ballot(hi == top && lo == low);
  }
  return __ffsll((long long)who) - 1;
}

__device__ __forceinline__ double lane_value(double v, int lane) {
  const u64 b = (u64)__double_as_longlong(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
  return __longlong_as_double((long long)((u64)hi << 32 | lo));
}

// What the lanes of a token do together: a row of 16 or a whole wave.
template <int LANES> struct Lanes;
template <> struct Lanes<64> {
  static __device__ __forceinline__ float largest(float v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
  }
  static __device__ __forceinline__ double sum(double v) { return wave_sum(v); }
  static __device__ __forceinline__ bool any(bool b) { return __ballot(b) != 0; }
  // The lane (of the token's) that holds the largest of their keys, the lowest one among
  // equals: lanes hold ascending experts.
  static __device__ __forceinline__ int best(u64 key) { return best_lane(key); }
  static __device__ __forceinline__ uint32_t largest_word(uint32_t v) { return wave_max(v); }
  // The lanes of `who` (some of the token's own at least): whether there are several of any
  // token's, and the lowest of this one's.
  static __device__ __forceinline__ bool several(u64 who) { return (who & (who - 1)) != 0; }
  static __device__ __forceinline__ int lowest(u64 who) { return __ffsll((long long)who) - 1; }
};
template <> struct Lanes<16> {
  // (rotations of the row: every lane ends with the whole)
  template <int N>
  static __device__ __forceinline__ uint32_t turn(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + N, 0xf, 0xf, true);
  }
  static __device__ __forceinline__ uint32_t largest_word(uint32_t v) {
    v = max(v, turn<8>(v));
    v = max(v, turn<4>(v));
    v = max(v, turn<2>(v));
    return max(v, turn<1>(v));
  }
  template <int N>
  static __device__ __forceinline__ float turn(float v) {
    return __uint_as_float(turn<N>(__float_as_uint(v)));
  }
  static __device__ __forceinline__ float largest(float v) {
    v = fmaxf(v, turn<8>(v));
    v = fmaxf(v, turn<4>(v));
    v = fmaxf(v, turn<2>(v));
    return fmaxf(v, turn<1>(v));
  }
  template <int N>
  static __device__ __forceinline__ double turn(double v) {
    const u64 b = (u64)__double_as_longlong(v);
    return __longlong_as_double((long long)((u64)turn<N>((uint32_t)(b >> 32)) << 32 | turn<N>((uint32_t)b)));
  }
  // (the same bits in every lane: a sum of two is the same either way round)
  static __device__ __forceinline__ double sum(double v) {
    v += turn<8>(v);
    v += turn<4>(v);
    v += turn<2>(v);
    return v + turn<1>(v);
  }
  static __device__ __forceinline__ uint32_t mine(u64 mask) { return (uint32_t)(mask >> (threadIdx.x & 48)) & 0xffffu; }
  static __device__ __forceinline__ bool any(bool b) { return mine(__ballot(b)) != 0; }
  static __device__ __forceinline__ bool several(u64 who) { return (who & (who - 0x0001000100010001ull)) != 0; }
  static __device__ __forceinline__ int lowest(u64 who) { return __ffs((int)mine(who)) - 1; }
  static __device__ __forceinline__ int best(u64 key) {
    const uint32_t hi = (uint32_t)(key >> 32), top = largest_word(hi);
    u64 who = __ballot(hi == top);
    if (several(who)) {
      const uint32_t lo = hi == top ? (uint32_t)key : 0u, low = largest_word(lo);
      who = __ballot(hi == top && lo == low);
    }
    return lowest(who);
  }
};

// V neighbouring elements of a row from e0 on, `other` beyond its end.
template <class L, int V>
__device__ __forceinline__ void load_neighbours(const L* row, int left, float other, float (&l)[V]) {
  if constexpr (V >= Vec<L>::N) {
    constexpr int N = Vec<L>::N;
    Vec<L> v[V / N];
#pragma unroll
    for (int h = 0; h < V / N; ++h)
      v[h] = left > h * N ? load_row(row + h * N, left - h * N) : Vec<L>{};
#pragma unroll
    for (int i = 0; i < V; ++i) l[i] = i < left ? v[i / N].get(i % N) : other;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) l[i] = i < left ? Elem<L>::to_f32(row[i]) : other;
  }
}

// Scores of the V experts from e0 on of a lane from their logits (those beyond the last: 0).
template <class L, int V, int LANES>
__device__ __forceinline__ void scores_of(const L* row, int experts, bool sigmoid, int e0, double (&s)[V]) {
  typedef Lanes<LANES> G;
  float l[V];
  load_neighbours<L, V>(row + e0, experts - e0, -INFINITY, l);
  if (sigmoid) {
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = 1.0 / (1.0 + exp(-(double)l[i]));  // (beyond the last: 0)
    return;
  }
  float big = -INFINITY;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    big = fmaxf(big, l[i]);
    nan |= l[i] != l[i];
  }
  big = G::largest(big);
  if (G::any(nan)) big = __uint_as_float(0x7fc00000u);  // the row's scores are NaN then
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    // (a row of -inf alone has no scores: zeros, not 0 / 0)
    s[i] = big != -INFINITY ? exp((double)l[i] - (double)big) : 0.0;  // (beyond the last: 0)
    sum += s[i];
  }
  sum = G::sum(sum);
#pragma unroll
  for (int i = 0; i < V; ++i) s[i] = big == -INFINITY ? 0.0 : s[i] / sum;
}

// LDS of a token: its scores, in whole lanes (before them, where a group's experts are not whole
// lanes', its c), and what it chose.
struct Stage {
  double* score;
  int* expert;
};

// Groups of `size` experts that are whole lanes, a power of two of them: their bounds are lanes'.
__device__ __forceinline__ bool whole_lanes(int size, int v) { return size % v == 0 && (size / v & (size / v - 1)) == 0; }

// One more to the two largest; the two largest of two pairs.
__device__ __forceinline__ void enter(double& first, double& second, double c) {
  const double low = fmin(first, c);
  first = fmax(first, c);
  second = fmax(second, low);
}
__device__ __forceinline__ void merge(double& first, double& second, double a, double b) {
  const double low = fmin(first, a);
  first = fmax(first, a);
  second = fmax(low, fmax(second, b));
}

// A token's choice to its stage, experts and scores in their order.
template <class L, int V, int LANES>
__device__ __forceinline__ void choose(const RouteArgs& a, int64_t t, const Stage& stage) {
  typedef Lanes<LANES> G;
  int lane = threadIdx.x & (LANES - 1);
  asm volatile("" : "+v"(lane));  // (what hangs on it is done where it is needed, not before the loop over tokens)
  const int e0 = lane * V;
  double s[V];
  scores_of<L, V, LANES>((const L*)a.logits + t * a.ldl, a.experts, a.sigmoid, e0, s);
  uint32_t hi[V], lo[V];  // of the experts' keys; hi 0: not to be chosen
  float bias[V];
#pragma unroll
  for (int i = 0; i < V; ++i) bias[i] = 0.0f;
  if (a.bias != nullptr) load_neighbours<float, V>(a.bias + e0, a.experts - e0, 0.0f, bias);
  const int size = a.experts / a.groups, span = size / V;  // experts and lanes of a group
  const bool whole = whole_lanes(size, V);
  double first = -INFINITY, second = -INFINITY;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const bool in = i < a.experts - e0;
    double c = a.bias != nullptr ? s[i] + (double)bias[i] : s[i];
    if (c != c) c = -INFINITY;  // a NaN counts as the lowest value
    const u64 key = key_of(c);
    hi[i] = in ? (uint32_t)(key >> 32) : 0u;
    lo[i] = (uint32_t)key;
    if (a.groups > 1) {
      if (whole)
        enter(first, second, c);  // (lanes beyond the last expert are no group's)
      else
        stage.score[e0 + i] = c;
    }
  }
  if (a.groups > 1) {
    const u64 none = 0;
    if (whole) {
      for (int d = 1; d < span; d <<= 1) merge(first, second, __shfl_xor(first, d), __shfl_xor(second, d));
      u64 rank = (lane & (span - 1)) == 0 && e0 < a.experts ? key_of(size > 1 ? first + second : first) : none;
      bool kept = false;
      for (int j = 0; j < a.top_groups; ++j) {
        const int g = G::best(rank);
        kept |= lane / span == g / span;
        if (lane == g) rank = none;
      }
#pragma unroll
      for (int i = 0; i < V; ++i) hi[i] = kept ? hi[i] : 0u;
    } else {
      // A lane takes a group (lanes of a row: every 16th); its experts are read from a place of its
      // own on, so that the lanes' reads spread over the banks.
      __builtin_amdgcn_wave_barrier();
      constexpr int N = kMaxGroups / LANES;
      u64 rank[N], kept = 0;
#pragma unroll
      for (int h = 0; h < N; ++h) {
        const int g = lane + h * LANES;
        first = second = -INFINITY;
        int j = lane % size;
        for (int i = 0; i < size && g < a.groups; ++i) {
          enter(first, second, stage.score[g * size + j]);
          j = j + 1 == size ? 0 : j + 1;
        }
        rank[h] = g < a.groups ? key_of(size > 1 ? first + second : first) : none;
      }
      __builtin_amdgcn_wave_barrier();
      for (int j = 0; j < a.top_groups; ++j) {
        u64 best = rank[0];
        int at = 0;
#pragma unroll
        for (int h = 1; h < N; ++h)
          if (rank[h] > best) {
            best = rank[h];
            at = h;
          }
        // groups ascend by h first: of equal ones the lowest h counts, then the lane
        int g = lane + at * LANES;
        if constexpr (N > 1) {
          const int l = G::best(best);
          const u64 most = __shfl(best, (threadIdx.x & 63 & ~(LANES - 1)) + l);
          int low = best == most ? g : kMaxGroups;
#pragma unroll
          for (int d = LANES / 2; d > 0; d >>= 1) low = min(low, __shfl_xor(low, d));
          if (g == low && best == most) {
#pragma unroll
            for (int h = 0; h < N; ++h)
              if (h == at) rank[h] = none;
          }
          g = low;
        } else {
          g = G::best(best);
          if (lane == g) rank[0] = none;
        }
        kept |= u64(1) << g;
      }
      int g = e0 / size, in = e0 - g * size;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (!(kept >> min(g, kMaxGroups - 1) & 1)) hi[i] = 0u;
        g += ++in == size;
        in = in == size ? 0 : in;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) stage.score[e0 + i] = s[i];
  auto largest = [&]() {
    uint32_t m = hi[0];
#pragma unroll
    for (int i = 1; i < V; ++i) m = max(m, hi[i]);
    return m;
  };
  uint32_t most = largest();
  for (int j = 0; j < a.top; ++j) {
    // By the high words alone, unless they leave several lanes, or several of a lane's experts
    const uint32_t top = G::largest_word(most);
    u64 who = __ballot(most == top);
    int at = 0, same = 0;
#pragma unroll
    for (int i = V - 1; i >= 0; --i) {
      const bool is = hi[i] == top;
      at = is ? i : at;
      same += is;
    }
    if (G::several(who) || __ballot(same > 1) != 0) {
      u64 best = 0;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const u64 key = (u64)hi[i] << 32 | lo[i];
        if (hi[i] != 0 && key > best) {
          best = key;
          at = i;
        }
      }
      who = u64(1) << ((threadIdx.x & 63 & ~(LANES - 1)) + G::best(best));
    }
    if (lane == G::lowest(who)) {
      stage.expert[j] = e0 + at;
#pragma unroll
      for (int i = 0; i < V; ++i) hi[i] = i == at ? 0u : hi[i];
      most = largest();
    }
  }
  __builtin_amdgcn_wave_barrier();  // (a wave's LDS accesses are served in order)
}

// Tokens t0 on, one for each LANES lanes of a wave (those from `end` on: none): weights and
// experts; `count`: LDS numbers of the experts' slots, or null.
template <class L, int V, int LANES>
__device__ __forceinline__ void route_tokens(const RouteArgs& a, int64_t t0, int64_t end, const Stage& stage, int* count) {
  typedef Lanes<LANES> G;
  const int lane = threadIdx.x & (LANES - 1);
  const int64_t t = t0 + (threadIdx.x & 63) / LANES;
  const bool there = t < end, live = there && (a.mask == nullptr || a.mask[t] != 0);
  // (a token that is not there is routed as the last one that is, to no effect)
  choose<L, V, LANES>(a, there ? t : end - 1, stage);
  int e = -1;
  double s = 0.0;
  if (live && lane < a.top) {
    e = stage.expert[lane];
    s = stage.score[e];
  }
  double w = s;
  if (a.renormalise) {
    const double sum = G::sum(s);
    w = sum == 0.0 ? 0.0 : s / sum;
  }
  if (there && lane < a.top) {
    a.weights[t * a.top + lane] = (float)(w * a.scale);
    a.chosen[t * a.top + lane] = e;
    if (count != nullptr && e >= 0) atomicAdd(&count[e], 1);  // (LDS; sums of ones in any order)
  }
}

// ---------------------------------------------------------------- the sort
// Whether expert e takes slots: anything else is in no row.
__device__ __forceinline__ bool taken(int e, int experts) { return (unsigned)e < (unsigned)experts; }

// Slots s0 .. s1 - 1 to their rows.  count: WAVES x experts numbers of LDS;
// first(e): the first row of this chunk's slots of expert e.
template <int WAVES, class First>
__device__ __forceinline__ void place_slots(const RouteArgs& a, int64_t s0, int64_t s1, int* count, First first) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tid = threadIdx.x;
  const int64_t per = ((s1 - s0 + WAVES - 1) / WAVES + 63) / 64 * 64;
  const int64_t b0 = min(s1, s0 + wave * per), b1 = min(s1, b0 + per);
  for (int i = tid; i < WAVES * a.experts; i += 64 * WAVES) count[i] = 0;
  __syncthreads();
  int* mine = count + wave * a.experts;
  for (int64_t s = b0 + lane; s < b1; s += 64) {
    const int e = a.chosen[s];
    if (taken(e, a.experts)) atomicAdd(&mine[e], 1);  // (LDS; sums of ones in any order)
  }
  __syncthreads();
  for (int e = tid; e < a.experts; e += 64 * WAVES) {
    int row = first(e);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const int c = count[w * a.experts + e];
      count[w * a.experts + e] = row;
      row += c;
    }
  }
  __syncthreads();
  const int bits = 32 - __clz(a.experts);  // of 0 .. experts
  volatile int* next = mine;
  for (int64_t s = b0; s < b1; s += 64) {
    int e = s + lane < b1 ? a.chosen[s + lane] : -1;
    const bool in = taken(e, a.experts);
    e = in ? e : a.experts;
    u64 same = ~u64(0);
    for (int b = 0; b < bits; ++b) {
      const u64 one = __ballot(e >> b & 1);
      same &= e >> b & 1 ? one : ~one;
    }
    const u64 before = same & ((u64(1) << lane) - 1);
    int row = -1;
    if (in) row = next[e] + __popcll(before);
    __builtin_amdgcn_wave_barrier();
    if (in && before == 0) next[e] = row + __popcll(same);
    __builtin_amdgcn_wave_barrier();
    if (s + lane < b1) {
      a.place[s + lane] = row;
      if (in) a.order[row] = (int32_t)(s + lane);
    }
  }
}

// Exclusive sums of the experts' totals by THREADS threads: start[e], start[experts] the
// total.  Up to kMaxExperts / THREADS neighbours a thread; sums: a number a wave.
template <int THREADS, class Total>
__device__ __forceinline__ void starts(int experts, int* start, int* sums, Total total) {
  constexpr int N = (kMaxExperts + THREADS - 1) / THREADS;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int v[N], sum = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = tid * N + i;
    v[i] = e < experts ? total(e) : 0;
    sum += v[i];
  }
  int run = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int up = __shfl_up(run, d);
    if (lane >= d) run += up;
  }
  if (lane == 63) sums[wave] = run;
  __syncthreads();
  int at = run - sum;
  for (int w = 0; w < wave; ++w) at += sums[w];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = tid * N + i;
    if (e < experts) start[e] = at;
    at += v[i];
    if (e == experts - 1) start[experts] = at;
  }
  __syncthreads();
}

constexpr int kRouteWaves = 8, kPlaceWaves = 4;
constexpr int kChunks = 512;      // most, and most numbers a wave of k_scan sums: 8 a lane
constexpr int64_t kFewSlots = 512;  // one workgroup does all of them
constexpr int64_t kFewTokens = 64;

// Tokens of a chunk.
__host__ __device__ inline int64_t chunk_tokens(int64_t tokens) {
  const int64_t least = (tokens + kChunks - 1) / kChunks;
  return least < kRouteWaves ? kRouteWaves : least;
}

// LDS of the choosing waves: scores, then choices.
__host__ __device__ inline size_t stage_bytes(int waves, int lanes, int v, int top) {
  return (size_t)waves * (64 / lanes) * ((size_t)lanes * v * 8 + (size_t)top * 4);
}
template <int LANES, int V>
__device__ __forceinline__ Stage stage_of(char* lds, int waves, int top) {
  const int tokens = waves * (64 / LANES), k = threadIdx.x / LANES;
  return {(double*)lds + k * (LANES * V), (int*)((double*)lds + tokens * (LANES * V)) + k * top};
}

// CHOOSE: route the chunk's tokens; else their experts are there.  counts: experts x
// chunks (null: no sort).
template <class L, int V, int LANES, bool CHOOSE>
__global__ __launch_bounds__(64 * kRouteWaves, 4) void k_route(RouteArgs a, int64_t per, int* counts) {
  extern __shared__ __align__(16) char lds[];
  int* count = (int*)(lds + (CHOOSE ? stage_bytes(kRouteWaves, LANES, V, a.top) : 0));
  const int64_t t0 = blockIdx.x * per, t1 = min(a.tokens, t0 + per);
  if (counts != nullptr) {
    for (int i = threadIdx.x; i < a.experts; i += 64 * kRouteWaves) count[i] = 0;
    __syncthreads();
  }
  if (CHOOSE) {
    const Stage stage = stage_of<LANES, V>(lds, kRouteWaves, a.top);
    constexpr int kEach = 64 / LANES;
    for (int64_t t = t0 + (threadIdx.x >> 6) * kEach; t < t1; t += kRouteWaves * kEach)
      route_tokens<L, V, LANES>(a, t, t1, stage, counts != nullptr ? count : nullptr);
  } else {
    for (int64_t s = t0 * a.top + threadIdx.x; s < t1 * a.top; s += 64 * kRouteWaves) {
      const int e = a.chosen[s];
      if (taken(e, a.experts)) atomicAdd(&count[e], 1);
    }
  }
  if (counts == nullptr) return;
  __syncthreads();
  for (int e = threadIdx.x; e < a.experts; e += 64 * kRouteWaves)
    counts[(int64_t)e * gridDim.x + blockIdx.x] = count[e];
}

// Each expert's counts by chunk to the sums before them, and its total.
__global__ __launch_bounds__(256) void k_scan(int* counts, int* totals, int experts, int chunks) {
  const int e = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (e >= experts) return;
  int* c = counts + (int64_t)e * chunks;
  constexpr int N = kChunks / 64;
  int v[N], sum = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = lane * N + i < chunks ? c[lane * N + i] : 0;
    sum += v[i];
  }
  int run = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int up = __shfl_up(run, d);
    if (lane >= d) run += up;
  }
  int at = run - sum;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (lane * N + i < chunks) c[lane * N + i] = at;
    at += v[i];
  }
  if (lane == 63) totals[e] = at;
}

__global__ __launch_bounds__(64 * kPlaceWaves) void k_place(RouteArgs a, int64_t per, const int* counts, const int* totals) {
  extern __shared__ int count[];
  __shared__ int start[kMaxExperts + 1], sums[kPlaceWaves];
  starts<64 * kPlaceWaves>(a.experts, start, sums, [&](int e) { return totals[e]; });
  const int64_t slots = a.tokens * a.top;
  if (blockIdx.x == 0)
    for (int e = threadIdx.x; e <= a.experts; e += 64 * kPlaceWaves) a.offsets[e] = start[e];
  // rows that no slot takes
  for (int64_t p = start[a.experts] + (int64_t)blockIdx.x * (64 * kPlaceWaves) + threadIdx.x; p < slots;
       p += (int64_t)gridDim.x * (64 * kPlaceWaves))
    a.order[p] = -1;
  const int64_t s0 = blockIdx.x * per * a.top, s1 = min(slots, s0 + per * a.top);
  place_slots<kPlaceWaves>(a, s0, s1, count,
                           [&](int e) { return start[e] + counts[(int64_t)e * gridDim.x + blockIdx.x]; });
}

// Few tokens: all of it in one workgroup.
template <class L, int V, int LANES, bool CHOOSE>
__global__ __launch_bounds__(512) void k_route_few(RouteArgs a) {
  extern __shared__ __align__(16) char lds[];
  int* count = (int*)(lds + (CHOOSE ? stage_bytes(8, LANES, V, a.top) : 0));
  __shared__ int start[kMaxExperts + 1], sums[8];
  if (CHOOSE) {
    const Stage stage = stage_of<LANES, V>(lds, 8, a.top);
    constexpr int kEach = 64 / LANES;
    for (int64_t t = (threadIdx.x >> 6) * kEach; t < a.tokens; t += 8 * kEach)
      route_tokens<L, V, LANES>(a, t, a.tokens, stage, nullptr);
    if (a.order == nullptr) return;
    __threadfence_block();  // the experts are read by other waves from here on
  }
  for (int e = threadIdx.x; e < a.experts; e += 512) count[e] = 0;
  __syncthreads();
  const int slots = (int)(a.tokens * a.top);
  for (int s = threadIdx.x; s < slots; s += 512) {
    const int e = a.chosen[s];
    if (taken(e, a.experts)) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  starts<512>(a.experts, start, sums, [&](int e) { return count[e]; });
  for (int e = threadIdx.x; e <= a.experts; e += 512) a.offsets[e] = start[e];
  for (int p = start[a.experts] + threadIdx.x; p < slots; p += 512) a.order[p] = -1;
  place_slots<8>(a, 0, slots, count, [&](int e) { return start[e]; });
}

// --------------------------------------------------------------- gradient
// A wave a token.  d = gradient of each score (zeros but for the chosen), then
// softmax: dl = s (d - sum s d), sigmoid: dl = d s sigmoid(-l), in 64 bits.  Of one
// expert far ahead of the others, m, d_m - sum s d cancels to what the others' scores leave
// (and so does the gradient of its renormalised weight).  As the s sum to one, it is
//   d_i - sum_k s_k d_k = (d_i - d_m) + sum_k s_k (d_m - d_k)
// for any d_m; with m the score above one half, or d_m = 0 where there is none, no
// term is larger than what it is off by matters.  (A single chosen expert's renormalised
// weight is one whatever its logits: its gradient comes out as zero.)  Under sigmoid
// only the chosen logits are read: the others' gradients are zeros.  Bound by instructions in 64 bits: 16384
// tokens, 8 of 256, renormalised or not, softmax 23 and 20 us, sigmoid 14 and 12.
template <class L, int V>
__global__ __launch_bounds__(256) void k_route_grad(RouteGradArgs a) {
  const int lane = threadIdx.x & 63, e0 = lane * V;
  for (int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); t < a.tokens; t += (int64_t)gridDim.x * 4) {
    const L* row = (const L*)a.logits + t * a.ldl;
    // lane j has the j-th choice: the gradient of its weight, and its score w
    int e = -1;
    double dw = 0.0, w = 0.0, slope = 1.0;
    if (lane < a.top) {
      e = a.chosen[t * a.top + lane];
      if (taken(e, a.experts)) dw = (double)a.dweights[t * a.top + lane] * a.scale;
      else e = -1;
    }
    // A token that takes no expert has no gradient, whatever its logits hold (a padded one's may be NaN)
    const bool idle = __ballot(e >= 0) == 0;
    double s[V], d[V];
    if (a.sigmoid) {
      // 1 - w as exp(-l) w: the difference would lose what w has lost to its rounding, from l = 21
      // on more than fp32's, from 37 on all of it
      if (e >= 0) {
        const double x = exp(-(double)Elem<L>::to_f32(row[e]));
        w = 1.0 / (1.0 + x);
        slope = x == INFINITY ? 0.0 : x * w * w;
      }
    } else {
      scores_of<L, V, 64>(row, a.experts, false, e0, s);
      if (a.renormalise) {
#pragma unroll
        for (int i = 0; i < V; ++i) {  // (the lane's choice lies with lane e / V)
          const double v = __shfl(s[i], e < 0 ? 0 : e / V);
          if (e >= 0 && e % V == i) w = v;
        }
      }
    }
    if (a.renormalise) {
      // d_j = (dw_j - sum dw w) / sum, w over sum, that of the chosen scores
      const double sum = wave_sum(w);
      w /= sum;
      const u64 ahead = __ballot(w > 0.5);
      const double most = ahead != 0 ? lane_value(dw, __ffsll((long long)ahead) - 1) : 0.0;
      const double dot = wave_sum(w * (most - dw));
      dw = sum == 0.0 ? 0.0 : (dw - most + dot) / sum;
    }
    dw *= slope;
#pragma unroll
    for (int i = 0; i < V; ++i) d[i] = 0.0;
    for (int j = 0; j < a.top; ++j) {
      const int ej = __builtin_amdgcn_readlane(e, j);
      const double dj = lane_value(dw, j);
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (ej == e0 + i) d[i] += dj;
    }
    if (!a.sigmoid && !idle) {
      double most = 0.0, dot = 0.0;
      bool mine = false;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (s[i] > 0.5) {
          mine = true;
          most = d[i];
        }
      const u64 ahead = __ballot(mine);
      most = ahead != 0 ? lane_value(most, __ffsll((long long)ahead) - 1) : 0.0;
#pragma unroll
      for (int i = 0; i < V; ++i) dot += s[i] * (most - d[i]);
      dot = wave_sum(dot);
#pragma unroll
      for (int i = 0; i < V; ++i) d[i] = s[i] * (d[i] - most + dot);
    }
    L* out = (L*)a.dlogits + t * a.ldd;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (e0 + i < a.experts) out[e0 + i] = Elem<L>::from_f32((float)d[i]);
  }
}

// f(V) for the neighbours a lane holds of `experts`
template <class F>
hipError_t for_experts(int experts, F f) {
  if (experts <= 64) return f(std::integral_constant<int, 1>());
  if (experts <= 128) return f(std::integral_constant<int, 2>());
  if (experts <= 256) return f(std::integral_constant<int, 4>());
  if (experts <= 512) return f(std::integral_constant<int, 8>());
  return f(std::integral_constant<int, 16>());
}

bool few(int64_t tokens, int top) { return tokens <= kFewTokens && tokens * top <= kFewSlots; }
int chunks_of(int64_t tokens) { return (int)((tokens + chunk_tokens(tokens) - 1) / chunk_tokens(tokens)); }

bool fits(const RouteArgs& a) {
  return a.tokens > 0 && a.experts >= 1 && a.experts <= kMaxExperts && a.top >= 1 && a.top <= kMaxTop &&
         a.tokens * a.top <= (int64_t(1) << 30);
}

template <class L, int V, int LANES, bool CHOOSE>
hipError_t route_for(const RouteArgs& a, void* workspace, hipStream_t s) {
  const bool sort = a.order != nullptr;
  if (few(a.tokens, a.top)) {
    const size_t lds = (CHOOSE ? stage_bytes(8, LANES, V, a.top) : 0) + (size_t)8 * a.experts * 4;
    hipLaunchKernelGGL((k_route_few<L, V, LANES, CHOOSE>), dim3(1), dim3(512), lds, s, a);
    return hipGetLastError();
  }
  const int64_t per = chunk_tokens(a.tokens);
  const int chunks = chunks_of(a.tokens);
  if (sort && workspace == nullptr) return hipErrorInvalidValue;
  int *counts = sort ? (int*)workspace : nullptr, *totals = counts + (sort ? (size_t)chunks * a.experts : 0);
  const size_t lds = (CHOOSE ? stage_bytes(kRouteWaves, LANES, V, a.top) : 0) + (size_t)a.experts * 4;
  hipLaunchKernelGGL((k_route<L, V, LANES, CHOOSE>), dim3(chunks), dim3(64 * kRouteWaves), lds, s, a, per, counts);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !sort) return e;
  hipLaunchKernelGGL(k_scan, dim3((a.experts + 3) / 4), dim3(256), 0, s, counts, totals, a.experts, chunks);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL(k_place, dim3(chunks), dim3(64 * kPlaceWaves), (size_t)kPlaceWaves * a.experts * 4, s, a, per,
                     counts, totals);
  return hipGetLastError();
}

}  // namespace

size_t route_workspace(int64_t tokens, int experts, int top) {
  return few(tokens, top) ? 0 : ((size_t)chunks_of(tokens) + 1) * (size_t)experts * 4;
}

hipError_t launch_route(const RouteArgs& a, void* workspace, hipStream_t s) {
  if (!fits(a) || a.top > a.experts || a.groups < 1 || a.groups > kMaxGroups || a.experts % a.groups != 0 ||
      a.top_groups < 1 || a.top_groups > a.groups || a.top > a.top_groups * (a.experts / a.groups))
    return hipErrorInvalidValue;
  // rows of 16 lanes: up to 16 experts a lane, a lane for each choice
  if (a.experts <= 256 && a.top <= 16)
    return for_experts(4 * a.experts, [&](auto v) {
      constexpr int V = decltype(v)::value;
      return a.bf16 ? route_for<bf16_t, V, 16, true>(a, workspace, s) : route_for<float, V, 16, true>(a, workspace, s);
    });
  return for_experts(a.experts, [&](auto v) {
    constexpr int V = decltype(v)::value;
    return a.bf16 ? route_for<bf16_t, V, 64, true>(a, workspace, s) : route_for<float, V, 64, true>(a, workspace, s);
  });
}

hipError_t launch_order(const RouteArgs& a, void* workspace, hipStream_t s) {
  if (!fits(a) || a.order == nullptr) return hipErrorInvalidValue;
  return route_for<float, 1, 64, false>(a, workspace, s);
}

hipError_t launch_route_grad(const RouteGradArgs& a, hipStream_t s) {
  if (a.tokens <= 0 || a.experts < 1 || a.experts > kMaxExperts || a.top < 1 || a.top > kMaxTop) return hipErrorInvalidValue;
  const dim3 grid((uint32_t)std::min<int64_t>((a.tokens + 3) / 4, 1 << 16));
  return for_experts(a.experts, [&](auto v) {
    constexpr int V = decltype(v)::value;
    if (a.bf16)
      hipLaunchKernelGGL((k_route_grad<bf16_t, V>), grid, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((k_route_grad<float, V>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
  });
}

}  // namespace ff
