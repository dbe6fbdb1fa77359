// The products of a layer of experts and their gradients, on rows sorted by expert.
//
//   y_p = act(x W_e^T + b_e),  out_t = sum_j weight_tj y of the token's rows
//   g_p = dy_p act'(z_p),  dx_p = g_p W_e,  dW_e = sum_{p in e} g_p^T x_p,  db_e = sum g_p
//
// How many rows an expert has is known on the device alone.  A launch has workgroups
// enough for any split of its rows (rows / BM + experts rows of tiles); each finds its
// tile by a wave's prefix sum over the experts' counts, and those too many, and some
// that are always there, clear the rows that are in no expert.  Tiles are
// numbered expert by expert and spread over the XCDs by what is in use, so that those that
// share a weight share an L2.
#include <math.h>

#include <algorithm>
#include <initializer_list>

#include "ff_expert_kernels.hpp"
#include "ff_linear_tile.hpp"
#include "ff_q8.hpp"
#include "ff_tile_kn.hpp"
#include "ff_vec.hpp"

namespace ff {
namespace {

constexpr int kClearers = 16;  // workgroups there at least for rows in no expert

__device__ __forceinline__ int64_t bounded(int32_t v, int64_t rows) { return v < 0 ? 0 : min((int64_t)v, rows); }
// Rows of the batch that are in an expert: lo .. hi - 1.  (lo is not 0 where the experts are some of those that the
// rows are sorted by.)
struct Used {
  int64_t lo, hi;
  __device__ __forceinline__ bool has(int64_t row) const { return row >= lo && row < hi; }
};
__device__ __forceinline__ Used used_rows(const SlotRows& at) {
  if (at.offsets == nullptr) return {0, at.rows};
  const int64_t lo = bounded(at.offsets[0], at.rows);
  return {lo, max(lo, bounded(at.offsets[at.experts], at.rows))};
}
// An expert's rows: their number, and the first.
__device__ __forceinline__ int64_t expert_rows(const SlotRows& at, int e, int64_t& first) {
  if (at.offsets == nullptr) {
    first = 0;
    return at.rows;
  }
  first = bounded(at.offsets[e], at.rows);
  return max((int64_t)0, bounded(at.offsets[e + 1], at.rows) - first);
}
// The token that row p stands for, or -1.
__device__ __forceinline__ int64_t token_of(const SlotRows& at, int64_t p) {
  const int32_t slot = at.order[p];
  if (slot < 0 || slot >= at.rows) return -1;
  return slot / at.top;
}

struct GroupTile {
  int expert;
  int64_t row0;  // its first row
  int rows;      // from there on, of this expert
  uint32_t col;  // tile column
};

// The tile of workgroup w of `grid` among row tiles of bm rows and `cols` tile columns; false, with
// `extra` its number among those, for workgroups beyond the last tile.
__device__ __forceinline__ bool find_tile(const SlotRows& at, int bm, uint32_t cols, uint32_t w, uint32_t grid, GroupTile& g,
                                          uint32_t& extra, uint32_t& extras) {
  const int lane = threadIdx.x & 63, n = (at.experts + 63) / 64, e0 = lane * n;
  uint32_t sum = 0;  // (rows <= 2^24: 2^30 row tiles at most, whatever the offsets hold)
  for (int i = 0; i < n; ++i) {
    int64_t first;
    if (e0 + i < at.experts) sum += (uint32_t)((expert_rows(at, e0 + i, first) + bm - 1) / bm);
  }
  uint32_t run = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t up = __shfl_up(run, d);
    if (lane >= d) run += up;
  }
  const uint64_t total = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)run, 63) * cols;
  const uint32_t used = (uint32_t)min(total, (uint64_t)grid);
  if (w >= used) {
    extra = w - used;
    extras = grid - used;
    return false;
  }
  const uint32_t t = xcd_remap(w, used);
  // the lane whose experts hold tile t, and which of them
  const bool mine = t >= (uint64_t)(run - sum) * cols && t < (uint64_t)run * cols;
  int expert = 0, rows = 0;
  int64_t row0 = 0;
  uint32_t in = 0;
  if (mine) {
    uint32_t before = run - sum;
    for (int i = 0; i < n; ++i) {
      int64_t first;
      if (e0 + i >= at.experts) break;
      const int64_t count = expert_rows(at, e0 + i, first);
      const uint32_t tiles = (uint32_t)((count + bm - 1) / bm);
      if (t < (uint64_t)(before + tiles) * cols) {
        expert = e0 + i;
        rows = (int)count;
        row0 = first;
        in = t - before * cols;
        break;
      }
      before += tiles;
    }
  }
  const int who = __ffsll((long long)__ballot(mine)) - 1;
  expert = __builtin_amdgcn_readlane(expert, who);
  rows = __builtin_amdgcn_readlane(rows, who);
  row0 = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)row0, who);
  in = (uint32_t)__builtin_amdgcn_readlane((int)in, who);
  uint32_t ti, tj;
  tile_at(in, (uint32_t)((rows + bm - 1) / bm), cols, ti, tj);
  g.expert = expert;
  g.row0 = row0 + (int64_t)ti * bm;
  g.rows = rows - (int)ti * bm;
  g.col = tj;
  return true;
}

// Rows in no expert, of `cols` elements, `ld` apart, are set to zeros.
template <class E>
__device__ __forceinline__ void clear_rows(const SlotRows& at, E* p, int64_t ld, int64_t cols, uint32_t extra,
                                           uint32_t extras) {
  const Used used = used_rows(at);
  for (int64_t i = extra; i < used.lo + at.rows - used.hi; i += extras) {
    const int64_t r = i < used.lo ? i : i - used.lo + used.hi;
    for (int64_t c = threadIdx.x; c < cols; c += blockDim.x) p[r * ld + c] = E(0);
  }
}

// The arguments of expert e's rows.
__device__ __forceinline__ LinearArgs args_of(const ExpertArgs& x, const GroupTile& g) {
  LinearArgs a{};
  const int64_t row0 = g.row0;
  a.tokens = g.rows;
  a.n = x.lin.n;
  a.m = x.lin.m;
  a.x = x.gather ? x.lin.x : (const bf16_t*)x.lin.x + row0 * x.lin.ldx;
  a.ldx = x.lin.ldx;
  a.w = (const bf16_t*)x.lin.w + (int64_t)g.expert * x.lin.m * x.lin.ldw;
  a.ldw = x.lin.ldw;
  a.bias = x.lin.bias != nullptr ? x.lin.bias + (int64_t)g.expert * x.lin.m : nullptr;
  a.y = x.lin.y + row0 * x.lin.ldy;
  a.ldy = x.lin.ldy;
  a.preact = x.lin.preact != nullptr ? x.lin.preact + row0 * x.lin.ldz : nullptr;
  a.ldz = x.lin.ldz;
  a.act = x.lin.act;
  return a;
}
__device__ __forceinline__ void clear_outputs(const ExpertArgs& x, uint32_t extra, uint32_t extras) {
  clear_rows(x.at, x.lin.y, x.lin.ldy, x.lin.m, extra, extras);
  if (x.lin.preact != nullptr) clear_rows(x.at, x.lin.preact, x.lin.ldz, x.lin.m, extra, extras);
}

// An expert's last tile takes half the height where that holds its rows: of 64 experts
// with 256 rows in the mean a quarter of the tiles' rows were none (4096 -> 2048: 384 us, 372 so).
constexpr int half_of(int ti) { return ti >= 4 && ti % 4 == 0 ? ti / 2 : ti; }
constexpr int half_slots(int ti, int slots) { return ti == 8 ? 3 : slots; }

template <int TI, int TJ, int SLOTS, bool GATHER>
__global__ __launch_bounds__(nt::kThreads, (LinearTile<nt::Bf16, TI, TJ, SLOTS>::kWaves)) void k_expert_tile(
    ExpertArgs x, uint32_t cols) {
  typedef LinearTile<nt::Bf16, TI, TJ, SLOTS> L;
  typedef LinearTile<nt::Bf16, half_of(TI), TJ, half_slots(TI, SLOTS)> H;
  __shared__ union {
    typename L::Shared whole;
    typename H::Shared half;
  } all;
  GroupTile g;
  uint32_t extra, extras;
  if (!find_tile(x.at, L::G::BM, cols, blockIdx.x, gridDim.x, g, extra, extras)) {
    clear_outputs(x, extra, extras);
    return;
  }
  const LinearArgs a = args_of(x, g);
  const int64_t i0 = (int64_t)g.col * L::G::BN;
  if (half_of(TI) < TI && g.rows <= H::G::BM)
    H::template run<GATHER>(all.half, a, 0, i0, 0, 1, nullptr, x.at.order + g.row0, x.at.top, x.at.tokens);
  else
    L::template run<GATHER>(all.whole, a, 0, i0, 0, 1, nullptr, x.at.order + g.row0, x.at.top, x.at.tokens);
}

// Experts of few rows: 16 NT of them against 16 outputs a workgroup, k among its waves, W read once and
// straight to registers.  Bound by that read: one token's 8 experts, 4096 -> 2048 (134 MB), 23 us, 5.8 TB/s.
template <int NT, int RW, int WAVES, bool GATHER>
__global__ __launch_bounds__(64 * WAVES) void k_expert_skinny(ExpertArgs x, uint32_t cols) {
  __shared__ SkinnySums<nt::Bf16, NT, RW, WAVES> sh;
  GroupTile g;
  uint32_t extra, extras;
  if (!find_tile(x.at, 16 * NT, cols, blockIdx.x, gridDim.x, g, extra, extras)) {
    clear_outputs(x, extra, extras);
    return;
  }
  g.rows = min(g.rows, 16 * NT);
  const LinearArgs a = args_of(x, g);
  skinny_run<nt::Bf16, NT, RW, WAVES, GATHER>(sh, a, (int64_t)g.col * (16 * RW), x.at.order + g.row0, x.at.top,
                                              x.at.tokens);
}

// ---------------------------------------------------------------- combining
// Eight columns a thread; the token's rows one after the other, in fp32, always in the order of
// its choices.  Bound by memory: four fp32 rows of 4096 for each of 4096 tokens (302 MB) in 60 us, 5.0 TB/s;
// small ones by latency (37 tokens: 5 us).
template <bool F32>
__global__ __launch_bounds__(256) void k_combine(CombineArgs a, uint32_t per_row, int64_t total) {
  for (int64_t b = (int64_t)blockIdx.x * 256; b < total; b += (int64_t)gridDim.x * 256) {
    const int64_t r = b / per_row;
    const uint32_t c = (uint32_t)(b - r * per_row) + threadIdx.x;
    const int64_t t = r + c / per_row, col = (int64_t)(c % per_row) * 8;
    if (t >= a.at.tokens) continue;
    const int count = (int)min((int64_t)8, a.cols - col);
    float s[8];
    if (a.residual != nullptr) {
      const Vec<bf16_t> v = load_row(a.residual + t * a.ldr + col, count);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] = v.get(i);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] = 0.0f;
    }
    for (int j = 0; j < a.at.top; ++j) {
      const int64_t p = F32 && a.at.place == nullptr ? t : a.at.place[t * a.at.top + j];
      if (p < 0 || p >= a.at.rows) continue;
      if (F32) {
        for (int z = 0; z < a.parts; ++z) {
          const float* y = (const float*)a.y + z * a.part_stride + p * a.ldy + col;
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (count > 4 * h) {
              const Vec<float> v = load_row(y + 4 * h, count - 4 * h);
#pragma unroll
              for (int i = 0; i < 4; ++i) s[4 * h + i] += v.get(i);
            }
        }
      } else {
        const float w = a.at.weights != nullptr ? a.at.weights[t * a.at.top + j] : 1.0f;
        const Vec<bf16_t> v = load_row((const bf16_t*)a.y + p * a.ldy + col, count);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] += w * v.get(i);
      }
    }
    Vec<bf16_t> o;
    o.set(s);
    store_row(a.out + t * a.ldo + col, o, count);
  }
}

// A wave a row: the row's gradient and its weight's (2042 rows of 333: 6.3 us, latency).  A slot is in a row of an
// expert where place and order name each other: the wave of that row writes its weight's gradient, and
// the wave of number p zero for slot p where there is no such row, so that each is written once.
__global__ __launch_bounds__(256) void k_combine_grad(CombineGradArgs a) {
  const int lane = threadIdx.x & 63;
  const Used used = used_rows(a.at);
  for (int64_t p = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); p < a.at.rows; p += (int64_t)gridDim.x * 4) {
    const int32_t slot = used.has(p) ? a.at.order[p] : -1;
    const bool live = slot >= 0 && slot < a.at.rows;
    bool own = false;
    if (a.dweights != nullptr && lane == 0) {
      const int32_t place = a.at.place[p];
      if (!used.has(place) || a.at.order[place] != p) a.dweights[p] = 0.0f;
      own = live && a.at.place[slot] == p;
    }
    const int64_t t = live ? slot / a.at.top : 0;
    const float w = live ? a.at.weights[slot] : 0.0f;
    float dot = 0.0f;
    for (int64_t col = lane * 8; col < a.cols; col += 512) {
      const int count = (int)min((int64_t)8, a.cols - col);
      float f[8];
      if (live) {
        const Vec<bf16_t> d = load_row(a.dout + t * a.ldd + col, count);
        if (a.dweights != nullptr) {
          const Vec<bf16_t> y = load_row(a.y + p * a.ldy + col, count);
#pragma unroll
          for (int i = 0; i < 8; ++i) dot += d.get(i) * y.get(i);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = w * d.get(i);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = 0.0f;
      }
      if (a.dy != nullptr) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (count > 4 * h) {
            Vec<float> o;
            o.set(f + 4 * h);
            store_row(a.dy + p * a.lddy + col + 4 * h, o, count - 4 * h);
          }
      }
    }
    if (a.dweights != nullptr && live) {
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) dot += __shfl_xor(dot, d);
      if (own) a.dweights[slot] = dot;
    }
  }
}

// ------------------------------------------------------------ operands' rows
// 2^e that takes values up to `factor` times the peak to at most 2^15 (fp16 ends at
// 2^16): the inverse is exact too.  A peak of zero: 1.
__device__ __forceinline__ int peak_exponent(uint32_t bits, float factor) {
  const float big = __uint_as_float(bits) * factor;
  if (!(big > 0.0f)) return 0;
  int e;
  frexpf(fminf(big, 0x1p127f), &e);  // big < 2^e
  return min(15 - e, 126);
}
// The largest of the peaks, by a workgroup of 256; every thread has it.
__device__ __forceinline__ uint32_t peak_of(const uint32_t* peaks, uint32_t* red) {
  static_assert(kPeaks == 4 * 256, "four a thread");
  const u32x4 p = *reinterpret_cast<const u32x4*>(peaks + 4 * threadIdx.x);
  uint32_t v = max(max(p[0], p[1]), max(p[2], p[3]));
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = max(max(red[0], red[1]), max(red[2], red[3]));
  __syncthreads();
  return v;
}

struct RowsJobs {
  RowsArgs job[3];
  uint32_t end[3];  // first workgroup after the job
  int part_rows;    // of job 0's parts
};

// Pieces of eight columns, `n` of them in their row (0: no such row, zeros), zeros beyond
// them, times act'(z).  All of a kind's loads go out before the first is waited for.  ONCE: which
// activation it is is decided once, not for each number; k_rows needs 92 registers so, 78 otherwise.
template <bool ONCE, int U>
__device__ __forceinline__ void load_pieces(const RowsArgs& a, const int64_t (&row)[U], const int64_t (&col)[U],
                                            const int (&n)[U], float (&f)[U][8]) {
  int64_t from[U];
  int have[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    from[u] = row[u];
    have[u] = n[u];
    if (a.gather && n[u] > 0) {
      from[u] = token_of(a.at, row[u]);
      if (from[u] < 0) have[u] = 0;
    }
  }
  auto codes = [&](const Q8Rows& q, const int64_t (&r)[U], auto use) {
    uint32_t w[U][2];
    float scale[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      w[u][0] = w[u][1] = 0;
      scale[u] = 0.0f;
      if (have[u] > 0) {
        load_codes(q.q + r[u] * q.ldq + col[u], have[u], w[u]);
        scale[u] = q.scale[r[u] * q.lds + (col[u] >> q.shift)];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[8];
      values_of(w[u], scale[u], v);
#pragma unroll
      for (int i = 0; i < 8; ++i) use(u, i, i < have[u] ? v[i] : 0.0f);  // (a NaN scale)
    }
  };
  auto values = [&](const bf16_t* p, int64_t ld, const int64_t (&r)[U], auto use) {
    Vec<bf16_t> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      v[u].w = u32x4{0, 0, 0, 0};
      if (have[u] > 0) v[u] = load_row(p + r[u] * ld + col[u], have[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) use(u, i, v[u].get(i));
  };
  auto put = [&](int u, int i, float v) { f[u][i] = v; };
  if (a.src_q8.q != nullptr) {
    codes(a.src_q8, from, put);
  } else if (a.src_f32) {
    Vec<float> v[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        v[u][h].w = u32x4{0, 0, 0, 0};
        if (have[u] > 4 * h) v[u][h] = load_row((const float*)a.src + from[u] * a.lds + col[u] + 4 * h, have[u] - 4 * h);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) f[u][i] = v[u][i / 4].get(i % 4);
  } else {
    values((const bf16_t*)a.src, a.lds, from, put);
  }
  if (a.z_q8.q == nullptr && a.z == nullptr) return;
  auto slopes = [&](auto act) {
    auto slope = [&](int u, int i, float v) { f[u][i] *= act_slope(v, act); };
    if (a.z_q8.q != nullptr)
      codes(a.z_q8, row, slope);
    else
      values(a.z, a.ldz, row, slope);
  };
  if (!ONCE)
    slopes(a.act);
  else if (a.act == kActRelu)
    slopes(std::integral_constant<int, kActRelu>());
  else if (a.act == kActGelu)
    slopes(std::integral_constant<int, kActGelu>());
  else
    slopes(std::integral_constant<int, kActSilu>());
}

struct PeaksJobs {
  RowsArgs job[2];
  uint32_t* peaks[2];
};
template <class E>
__device__ __forceinline__ uint32_t peak_bits(const RowsArgs& a, int64_t block, int64_t blocks) {
  constexpr int N = Vec<E>::N, U = 2;  // (4: as fast for large arrays, 5.5 us instead of 4.6 for 1021 x 777)
  uint32_t big = 0;
  const uint32_t per_row = (uint32_t)((a.cols + N - 1) / N);
  const Used used = used_rows(a.at);
  const int64_t total = (used.hi - used.lo) * per_row;
  for (int64_t b = block * (256 * U); b < total; b += blocks * (256 * U)) {
    const int64_t r = b / per_row;
    Vec<E> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t c = (uint32_t)(b - r * per_row) + u * 256 + threadIdx.x;
      const int64_t col = (int64_t)(c % per_row) * N;
      int64_t row = used.lo + r + c / per_row;
      v[u].w = u32x4{0, 0, 0, 0};
      if (row < used.hi && (!a.gather || (row = token_of(a.at, row)) >= 0))
        v[u] = load_row((const E*)a.src + row * a.lds + col, a.cols - col);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const uint32_t bits = __float_as_uint(v[u].get(i)) & 0x7fffffffu;
        if (bits < 0x7f800000u) big = max(big, bits);
      }
  }
  return big;
}
// The same of dy act'(z): where the slope is zero, or next to it, dy may be far above all of g.  Bound by the
// slopes' instructions and the reads, hardly overlapped (4096 x 11008 of bf16 and codes, 137 MB, 50 us).
__device__ __forceinline__ uint32_t peak_bits_of_g(const RowsArgs& a, int64_t block, int64_t blocks) {
  constexpr int U = 2;
  uint32_t big = 0;
  const uint32_t per_row = (uint32_t)((a.cols + 7) / 8);
  const Used used = used_rows(a.at);
  const int64_t total = (used.hi - used.lo) * per_row;
  for (int64_t b = block * (256 * U); b < total; b += blocks * (256 * U)) {
    const int64_t r = b / per_row;
    int64_t row[U], col[U];
    int count[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t c = (uint32_t)(b - r * per_row) + u * 256 + threadIdx.x;
      row[u] = used.lo + r + c / per_row;
      col[u] = (int64_t)(c % per_row) * 8;
      count[u] = row[u] < used.hi ? (int)min((int64_t)8, a.cols - col[u]) : 0;
    }
    float f[U][8];
    load_pieces<true>(a, row, col, count, f);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(f[u][i]) & 0x7fffffffu);
      if (most >= 0x7f800000u) {  // (hardly ever: one by one)
        most = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t bits = __float_as_uint(f[u][i]) & 0x7fffffffu;
          if (bits < 0x7f800000u) most = max(most, bits);
        }
      }
      big = max(big, most);
    }
  }
  return big;
}
// The largest finite magnitudes of kPeaks parts of each array: no atomic, and no values to clear
// beforehand (4096 x 11008 of bf16, 90 MB, and the other operand's scales: 24 us, 3.8 TB/s).
__global__ __launch_bounds__(256) void k_peaks(PeaksJobs jobs) {
  __shared__ uint32_t red[4];
  const int which = blockIdx.x >= kPeaks;
  const RowsArgs& a = jobs.job[which];
  const int block = blockIdx.x % kPeaks;
  uint32_t big = a.z != nullptr || a.z_q8.q != nullptr ? peak_bits_of_g(a, block, kPeaks)
                 : a.src_f32                           ? peak_bits<float>(a, block, kPeaks)
                                                       : peak_bits<bf16_t>(a, block, kPeaks);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) big = max(big, (uint32_t)__shfl_xor((int)big, d));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = big;
  __syncthreads();
  if (threadIdx.x == 0) jobs.peaks[which][block] = max(max(red[0], red[1]), max(red[2], red[3]));
}

// Its outputs; the rounded values to `o`.
__device__ __forceinline__ void store_piece(const RowsArgs& a, int64_t row, int64_t col, int n, const float (&f)[8], float scale,
                                            Vec<bf16_t>& o) {
  const int64_t ldl = (a.cols + 7) / 8 * 8;
  o.set(f);
  if (a.out != nullptr) store_row(a.out + row * a.ldo + col, o, n);
  if (a.laid != nullptr) *reinterpret_cast<u32x4*>(a.laid + row * ldl + col) = o.w;
  if (a.scaled != nullptr) {
    u32x4 w;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      w[q] = (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)(f[2 * q] * scale)) |
             (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)(f[2 * q + 1] * scale)) << 16;
    *reinterpret_cast<u32x4*>(a.scaled + row * ldl + col) = w;
  }
}

// The operands of the gradients' products: g = dy act'(z) as the caller's rows, as bf16 rows of whole
// pieces and in fp16, and the sums of its columns; x and W as such rows.  All that a call needs are jobs of
// one launch.  Bound by memory (16384 x 2048 and, gathered, 16384 x 4096 from checkpoints: 390 MB in 97 to
// 106 us, 3.7 TB/s or more), small ones by latency (1021 x 777 and x 1000: 15 us).
template <bool ONCE>
__global__ __launch_bounds__(256) void k_rows(RowsJobs jobs) {
  __shared__ uint32_t red[4];
  __shared__ float sums[256][9];
  const int which = (blockIdx.x >= jobs.end[0]) + (blockIdx.x >= jobs.end[1]);
  const RowsArgs& a = jobs.job[which];
  const uint32_t first = which > 0 ? jobs.end[which - 1] : 0, blocks = jobs.end[which] - first, w = blockIdx.x - first;
  const uint32_t per_row = (uint32_t)((a.cols + 7) / 8);
  float scale = 1.0f;
  if (a.scaled != nullptr) {
    const int e = peak_exponent(peak_of(a.peaks, red), a.peak_factor);
    scale = ldexpf(1.0f, e);
    if (w == 0 && threadIdx.x == 0) *a.inverse = ldexpf(1.0f, -e);
  }
  if (a.parts != nullptr) {
    // Rows of one expert, part_rows at a time: 2^s threads across, their columns summed over the rows
    const int s = per_row >= 64 ? 6 : 32 - __clz((int)per_row - 1 | 1), down = 256 >> s;
    const int c = threadIdx.x & ((1 << s) - 1), r = threadIdx.x >> s;
    GroupTile g;
    uint32_t extra, extras;
    if (!find_tile(a.at, jobs.part_rows, (per_row + (1u << s) - 1) >> s, w, blocks, g, extra, extras)) {
      const int64_t ldl = (int64_t)per_row * 8;
      if (a.out != nullptr) clear_rows(a.at, a.out, a.ldo, a.cols, extra, extras);
      if (a.laid != nullptr) clear_rows(a.at, a.laid, ldl, ldl, extra, extras);
      if (a.scaled != nullptr) clear_rows(a.at, a.scaled, ldl, ldl, extra, extras);
      return;
    }
    const int64_t col = ((int64_t)(g.col << s) + c) * 8;
    const int n = (int)min((int64_t)8, max((int64_t)0, a.cols - col)), rows = min(g.rows, jobs.part_rows);
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
    constexpr int U = 2;  // rows a thread has in flight (4: 86 us where these take 73, 4096 x 11008 and x 4096)
    for (int k = r; n > 0 && k < rows; k += U * down) {
      float f[U][8];
      int64_t row[U], cols[U];
      int count[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        row[u] = g.row0 + k + u * down;
        cols[u] = col;
        count[u] = k + u * down < rows ? n : 0;
      }
      load_pieces<ONCE>(a, row, cols, count, f);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (count[u] > 0) {
          Vec<bf16_t> o;
          store_piece(a, row[u], col, n, f[u], scale, o);
#pragma unroll
          for (int i = 0; i < 8; ++i) sum[i] += o.get(i);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[threadIdx.x][i] = sum[i];
    __syncthreads();
    // (g.row0 is the expert's first row and a multiple of part_rows more)
    if (r == 0 && n > 0) {
      for (int k = 1; k < down; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += sums[(k << s) + c][i];
      float* p = a.parts + (g.row0 / jobs.part_rows + g.expert) * (int64_t)per_row * 8 + col;
      __builtin_memcpy(p, sum, 32);
    }
    return;
  }
  const int64_t total = a.at.rows * per_row;
  const Used used = used_rows(a.at);
  constexpr int U = 2;
  for (int64_t b = (int64_t)w * (256 * U); b < total; b += (int64_t)blocks * (256 * U)) {
    const int64_t r = b / per_row;
    float f[U][8];
    int64_t row[U], col[U];
    int count[U], have[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t c = (uint32_t)(b - r * per_row) + u * 256 + threadIdx.x;
      row[u] = r + c / per_row;
      col[u] = (int64_t)(c % per_row) * 8;
      count[u] = row[u] < a.at.rows ? (int)min((int64_t)8, a.cols - col[u]) : 0;
      have[u] = used.has(row[u]) ? count[u] : 0;
    }
    load_pieces<ONCE>(a, row, col, have, f);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Vec<bf16_t> o;
      if (count[u] > 0) store_piece(a, row[u], col[u], count[u], f[u], scale, o);
    }
  }
}

// ------------------------------------------------------------------ gradients
// The lane, counted where it is asked for: addresses of a tile's results would otherwise be kept through
// a loop over tiles, and spilled.
__device__ __forceinline__ int lane_here() {
  uint32_t none = 0;
  asm volatile("" : "+v"(none));
  return (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, none));
}

__device__ __forceinline__ int wave_here() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// What takes the sums of fp16 operands back is 2^e: one power of two for both, as the first of two
// factors alone may leave fp32's range where the result does not.
__device__ __forceinline__ int sums_exponent(const ExpertGradArgs& a) {
  if (!a.f16) return 0;
  const uint32_t g = __float_as_uint(a.inverse[0]) >> 23, x = __float_as_uint(a.inverse[1]) >> 23;
  return __builtin_amdgcn_readfirstlane((int)(g + x)) - 254;
}

// A tile of C, times 2^e, to its rows: `rows` and `cols` from the tile's corner on exist, E is
// bf16_t or float.  Each wave turns its own part over in its quarter of LDS that is free by then: a
// lane has four columns of a row, and writes 16 bytes beside its neighbours', whole lines of a
// row at once (8192 tiles of 256 x 256 with 256 rows each: 796 us with the lanes' own 8 bytes).
// 16-byte piece c of row r sits at c ^ (r & 15) of its row: 64 banks for either way.
template <class G, class E, class Free>
__device__ __forceinline__ void store_tile(Free& free, const typename G::Acc& acc, E* corner, int64_t ld, int64_t rows,
                                           int64_t cols, int e, int wave) {
  constexpr int TI = (int)(sizeof(typename G::Acc) / sizeof(f32x4[G::BN / 32])), TJ = G::BN / 32;
  constexpr int kLine = 16 * TJ * (int)sizeof(E), kPieces = kLine / 16, kPer = 16 / (int)sizeof(E);  // of a wave's row
  constexpr int kSwz = kPieces < 16 ? kPieces - 1 : 15;
  // tile rows of 16 a phase
  constexpr int kFit = (int)sizeof(Free) / 4 / (16 * kLine), H = kFit >= TI ? TI : kFit >= TI / 2 ? TI / 2 : 1;
  constexpr int kRows = 64 / kPieces;  // the wave stores at once
  static_assert(kFit >= 1 && TI % H == 0 && kPieces <= 64 && 16 * H % kRows == 0, "a wave's part of a phase");
  const int lane = lane_here();
  char* mine = reinterpret_cast<char*>(&free) + wave * (sizeof(Free) / 4);
  const int piece = lane % kPieces, col = (wave & 1) * 16 * TJ + piece * kPer;
  int row = (wave >> 1) * 16 * TI + lane / kPieces;
  asm volatile("" : "+s"(ld));  // (so would 32 rows' offsets)
  E* to_row = corner + row * ld + col;
#pragma unroll
  for (int h = 0; h < TI / H; ++h) {
#pragma unroll
    for (int i = 0; i < H; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j) {
        __builtin_amdgcn_sched_barrier(0);  // (read here, not all of them beforehand)
        const f32x4 a = acc[h * H + i][j];
        const float f[4] = {ldexpf(a[0], e), ldexpf(a[1], e), ldexpf(a[2], e), ldexpf(a[3], e)};
        const int r = i * 16 + (lane & 15), at = (16 * j + 4 * (lane >> 4)) * (int)sizeof(E);
        char* to = mine + r * kLine + (((at >> 4) ^ (r & kSwz)) << 4) + (at & 15);
        if constexpr (sizeof(E) == 4) {
          *reinterpret_cast<f32x4*>(to) = f32x4{f[0], f[1], f[2], f[3]};
        } else {
          typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
          *reinterpret_cast<u32x2*>(to) = u32x2{(uint32_t)f32_to_bf16(f[0]) | (uint32_t)f32_to_bf16(f[1]) << 16,
                                                (uint32_t)f32_to_bf16(f[2]) | (uint32_t)f32_to_bf16(f[3]) << 16};
        }
      }
    __builtin_amdgcn_wave_barrier();  // (a wave's LDS accesses are served in order)
#pragma unroll
    for (int q = 0; q < 16 * H / kRows; ++q) {
      const int r = q * kRows + lane / kPieces;
      Vec<E> o;
      o.w = *reinterpret_cast<const u32x4*>(mine + r * kLine + ((piece ^ (r & kSwz)) << 4));
      if (row < rows) store_row(to_row, o, cols - col);
      row += kRows;
      to_row += kRows * ld;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// The same for a whole tile of bf16 whose rows begin at 16 bytes: in a stream of tiles
// nothing else runs meanwhile, and the general way has a conversion and half a test more for each number
// (64 experts of 256 rows in the mean, 4096 x 2048, 256 x 256 a tile: 520 us, 484 so; 64 of 64 rows, 2048 x 1408, in
// tiles of 128: 120 and 101 with the scalar loads of stream_rows).
template <class G, class Free>
__device__ __forceinline__ void store_whole(Free& free, const typename G::Acc& acc, bf16_t* corner, int64_t ld, int e,
                                            int wave) {
  constexpr int TI = (int)(sizeof(typename G::Acc) / sizeof(f32x4[G::BN / 32])), TJ = G::BN / 32;
  constexpr int kLine = 32 * TJ, kPieces = kLine / 16, kSwz = kPieces - 1, kRows = 64 / kPieces;
  static_assert(sizeof(Free) / 4 >= 16 * kLine && kPieces <= 16, "a wave's part of a phase");
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
  const int lane = lane_here();
  char* mine = reinterpret_cast<char*>(&free) + wave * (sizeof(Free) / 4);
  const int r16 = lane & 15, piece = lane % kPieces, row = lane / kPieces, step = (int)(kRows * ld * 2);
  const uint32_t at = (uint32_t)(row * ld * 2) + 16u * (uint32_t)piece;
  const auto to = nt::rsrc((const char*)(corner + (int64_t)(wave >> 1) * 16 * TI * ld + (wave & 1) * 16 * TJ));
  // (rows are stored when the next ones' are on their way through LDS: a wave's accesses are served in order)
  constexpr int kEach = 16 / kRows;
  u32x4 o[2][kEach];
  int down = 0;
#pragma unroll
  for (int i = 0; i <= TI; ++i) {
    if (i < TI) {
#pragma unroll
      for (int j = 0; j < TJ; ++j) {
        __builtin_amdgcn_sched_barrier(0);  // (the sums are read here, not all of them beforehand)
        const f32x4 a = acc[i][j];
        const bf16x2 lo = __builtin_convertvector((f32x2{ldexpf(a[0], e), ldexpf(a[1], e)}), bf16x2);
        const bf16x2 hi = __builtin_convertvector((f32x2{ldexpf(a[2], e), ldexpf(a[3], e)}), bf16x2);
        const int b = 32 * j + 8 * (lane >> 4);
        *reinterpret_cast<u32x2*>(mine + r16 * kLine + (((b >> 4) ^ (r16 & kSwz)) << 4) + (b & 15)) =
            u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
      }
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int q = 0; q < kEach; ++q) {
        const int r = q * kRows + row;
        o[i & 1][q] = *reinterpret_cast<const u32x4*>(mine + r * kLine + ((piece ^ (r & kSwz)) << 4));
      }
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_sched_barrier(0);
    }
    if (i > 0)
#pragma unroll
      for (int q = 0; q < kEach; ++q) {
        __builtin_amdgcn_raw_buffer_store_b128(o[(i - 1) & 1][q], to, (int)at, down, 0);
        down += step;
      }
  }
}

// A tile of dx by workgroup w of `grid`, k in `splits` parts.  64 experts of 256 rows in the mean, 2048 x
// 4096, to fp32: 415 us (W_e is 1.1 GB, read from memory once; the products alone would take 173 us): ends of
// tiles, and experts' last ones that are not full.
template <int TI, int TJ, int SLOTS>
struct DxTile {
  typedef kn::Tile<nt::Bf16, false, TI, TJ, SLOTS> G;
  typedef kn::Tile<nt::Bf16, false, half_of(TI), TJ, half_slots(TI, SLOTS)> H;
  union Shared {
    typename G::Ring whole;
    typename H::Ring half;
  };
  static __device__ __forceinline__ void run(Shared& rings, const ExpertGradArgs& a, uint32_t cols, uint32_t splits, uint32_t w,
                                             uint32_t grid) {
    GroupTile g;
    uint32_t extra, extras;
    if (!find_tile(a.at, G::BM, cols * splits, w, grid, g, extra, extras)) {
      if (a.out_f32)
        for (uint32_t z = 0; z < splits; ++z) clear_rows(a.at, (float*)a.out + z * a.part_stride, a.ldo, a.n, extra, extras);
      else
        clear_rows(a.at, (uint16_t*)a.out, a.ldo, a.n, extra, extras);
      return;
    }
    const uint32_t z = g.col / cols;
    const int64_t n0 = (int64_t)(g.col - z * cols) * G::BN;
    const int64_t pairs = (a.m + kn::kK - 1) / kn::kK, k0 = pairs * z / splits * kn::kK;
    const int64_t k1 = min(a.m, pairs * (z + 1) / splits * kn::kK);
    const kn::Side P{(const char*)(a.g + g.row0 * a.ldg + k0), g.rows, (uint32_t)(a.ldg * 2)};
    const kn::Side Q{(const char*)(a.w + ((int64_t)g.expert * a.m + k0) * a.ldw + n0), a.n - n0, (uint32_t)(a.ldw * 2)};
    auto one = [&](auto& ring, auto tile) {
      typedef decltype(tile) T;
      typename T::Acc acc;
      T::zero(acc);
      T::loop(ring, P, Q, k1 - k0, acc);
      if (a.out_f32)
        store_tile<T>(ring, acc, (float*)a.out + z * a.part_stride + g.row0 * a.ldo + n0, a.ldo, g.rows, a.n - n0, 0, wave_here());
      else
        store_tile<T>(ring, acc, (bf16_t*)a.out + g.row0 * a.ldo + n0, a.ldo, g.rows, a.n - n0, 0, wave_here());
    };
    if (half_of(TI) < TI && g.rows <= H::BM)
      one(rings.half, H());
    else
      one(rings.whole, G());
  }
};

template <int TI, int TJ, int SLOTS>
__global__ __launch_bounds__(nt::kThreads, (DxTile<TI, TJ, SLOTS>::G::kWaves)) void k_expert_dx(ExpertGradArgs a, uint32_t cols,
                                                                                                uint32_t splits) {
  typedef DxTile<TI, TJ, SLOTS> D;
  __shared__ typename D::Shared rings;
  D::run(rings, a, cols, splits, blockIdx.x, gridDim.x);
}

// An expert's column sums from those of its parts: the column of each thread.
__device__ __forceinline__ void sum_column(const ExpertGradArgs& a, int64_t e, int64_t row0, int64_t rows, int64_t col) {
  const int64_t ld = (a.m + 7) / 8 * 8, first = row0 / a.part_rows + e, count = (rows + a.part_rows - 1) / a.part_rows;
  const float* p = a.parts + first * ld + col;
  float v = 0.0f;
#pragma unroll 8
  for (int64_t k = 0; k < count; ++k) v += p[k * ld];
  a.db[e * a.m + col] = f32_to_bf16(v);
}
__global__ __launch_bounds__(256) void k_expert_db(ExpertGradArgs a) {
  const int64_t col = (int64_t)blockIdx.x * 256 + threadIdx.x;
  int64_t row0;
  const int64_t rows = expert_rows(a.at, blockIdx.y, row0);
  if (col < a.m) sum_column(a, blockIdx.y, row0, rows, col);
}

// A tile of dW by workgroup w.  Every XCD takes an eighth of each expert's tiles: their work is the
// expert's rows, and with whole experts to an XCD the fullest one's kept the others waiting (8 experts of
// 422 to 2247 rows, 4096 x 4096: 480 us, 292 so).  The tiles of the first columns add up db as well.
template <class T, int TI, int TJ, int SLOTS>
struct DwTile {
  typedef kn::Tile<T, true, TI, TJ, SLOTS> G;
  static __device__ __forceinline__ void run(typename G::Ring& ring, const ExpertGradArgs& a, uint32_t mt, uint32_t ntl,
                                             uint32_t splits, uint32_t w) {
    const uint32_t tiles = mt * ntl * splits, share = (tiles + 7) / 8, local = w >> 3, e = local / share;
    const uint32_t tile = (w & 7) * share + (local - e * share);
    if (tile >= tiles) return;
    const uint32_t z = tile / (mt * ntl);
    uint32_t ti, tj;
    tile_at(tile - z * (mt * ntl), mt, ntl, ti, tj);
    const int64_t m0 = (int64_t)ti * G::BM, n0 = (int64_t)tj * G::BN;
    int64_t row0;
    const int64_t rows = expert_rows(a.at, (int)e, row0);
    const int64_t pairs = (rows + kn::kK - 1) / kn::kK, k0 = pairs * z / splits * kn::kK;
    const int64_t k1 = min(rows, pairs * (z + 1) / splits * kn::kK);
    const kn::Side P{(const char*)(a.g + (row0 + k0) * a.ldg + m0), a.m - m0, (uint32_t)(a.ldg * 2)};
    const kn::Side Q{(const char*)(a.x + (row0 + k0) * a.ldx + n0), a.n - n0, (uint32_t)(a.ldx * 2)};
    const int scale = sums_exponent(a);
    if (a.db != nullptr && tj == 0 && z == 0 && threadIdx.x < G::BM && m0 + threadIdx.x < a.m)
      sum_column(a, e, row0, rows, m0 + threadIdx.x);
    typename G::Acc acc;
    G::zero(acc);
    if (k1 > k0) G::loop(ring, P, Q, k1 - k0, acc);
    const int64_t at = ((int64_t)e * a.m + m0) * a.ldo + n0;
    if (a.out_f32)
      store_tile<G>(ring, acc, (float*)a.out + z * a.part_stride + at, a.ldo, a.m - m0, a.n - n0, scale, wave_here());
    else
      store_tile<G>(ring, acc, (bf16_t*)a.out + at, a.ldo, a.m - m0, a.n - n0, scale, wave_here());
  }
};

template <class T, int TI, int TJ, int SLOTS>
__global__ __launch_bounds__(nt::kThreads, (kn::Tile<T, true, TI, TJ, SLOTS>::kWaves)) void k_expert_dw(
    ExpertGradArgs a, uint32_t mt, uint32_t ntl, uint32_t splits) {
  typedef DwTile<T, TI, TJ, SLOTS> D;
  __shared__ typename D::G::Ring ring;
  D::run(ring, a, mt, ntl, splits, blockIdx.x);
}

// Both gradients in one launch where each alone would leave units empty (the smallest tiles; 1021 tokens,
// 1000 x 777: 9.5 and 13 us one after the other, 13.8 so).  The first `first` workgroups take dx.
template <class T, int TI, int TJ, int SLOTS>
__global__ __launch_bounds__(nt::kThreads, (kn::Tile<T, true, TI, TJ, SLOTS>::kWaves)) void k_expert_both(
    ExpertGradArgs x, uint32_t cols, uint32_t x_splits, uint32_t first, ExpertGradArgs w, uint32_t mt, uint32_t ntl,
    uint32_t w_splits) {
  typedef DxTile<TI, TJ, SLOTS> X;
  typedef DwTile<T, TI, TJ, SLOTS> W;
  __shared__ union {
    typename X::Shared x;
    typename W::G::Ring w;
  } sh;
  if (blockIdx.x < first)
    X::run(sh.x, x, cols, x_splits, blockIdx.x, first);
  else
    W::run(sh.w, w, mt, ntl, w_splits, blockIdx.x - first);
}

// ---------------------------------------------------------------------- host
constexpr int64_t kMaxSlots = int64_t(1) << 24, kMaxGrid = 0x7fffffff;

bool fits(const SlotRows& at) {
  return at.rows > 0 && at.rows <= kMaxSlots && at.top >= 1 && at.top <= kMaxTop && at.tokens * at.top == at.rows &&
         at.experts >= 1 && at.experts <= kMaxExperts && (at.offsets != nullptr || at.experts == 1);
}
// Workgroups for any split of the rows among the experts.
int64_t grid_for(const SlotRows& at, int64_t bm, int64_t cols) {
  return (at.rows / bm + std::min<int64_t>(at.experts, at.rows)) * cols + kClearers;
}

template <int TI, int TJ, int SLOTS>
hipError_t expert_tiles(const ExpertArgs& a, hipStream_t s) {
  typedef LinearTile<nt::Bf16, TI, TJ, SLOTS> L;
  const int64_t cols = (a.lin.m + L::G::BN - 1) / L::G::BN, grid = grid_for(a.at, L::G::BM, cols);
  if (grid > kMaxGrid) return hipErrorInvalidValue;
  if (a.gather)
    hipLaunchKernelGGL((k_expert_tile<TI, TJ, SLOTS, true>), dim3((uint32_t)grid), dim3(nt::kThreads), 0, s, a, (uint32_t)cols);
  else
    hipLaunchKernelGGL((k_expert_tile<TI, TJ, SLOTS, false>), dim3((uint32_t)grid), dim3(nt::kThreads), 0, s, a, (uint32_t)cols);
  return hipGetLastError();
}

template <int NT, int RW, int WAVES>
hipError_t expert_skinny(const ExpertArgs& a, hipStream_t s) {
  const int64_t cols = (a.lin.m + 16 * RW - 1) / (16 * RW), grid = grid_for(a.at, 16 * NT, cols);
  if (grid > kMaxGrid) return hipErrorInvalidValue;
  if (a.gather)
    hipLaunchKernelGGL((k_expert_skinny<NT, RW, WAVES, true>), dim3((uint32_t)grid), dim3(64 * WAVES), 0, s, a, (uint32_t)cols);
  else
    hipLaunchKernelGGL((k_expert_skinny<NT, RW, WAVES, false>), dim3((uint32_t)grid), dim3(64 * WAVES), 0, s, a, (uint32_t)cols);
  return hipGetLastError();
}

// Tiles in a stream (ff_tile_kn.hpp): with few rows an expert a tile is mostly starting,
// waiting for its first rows and storing, which the next tile's copies run beside.  Each XCD's
// workgroups, as many as its units hold, take the tiles of its eighth of every expert's in turn,
// experts by falling numbers of rows, so that all of them end alike (64 experts of 256 rows in the mean, 4096 x
// 2048: 484 us, one workgroup a tile 615; of 64 rows, 2048 x 1408 in tiles of 128: 101 and 132).  What is
// left (with parts of it left out in turn): 234 the loops of four pairs, 80 to 100 what their copies wait, 100 the
// stores' 1.1 GB, the rest their conversion.  Not waiting for a tile's stores before its next one's second pair changed
// nothing.
// (An expert's rows by scalar loads: a vector load would be waited for together with the copies and stores on
// their way, twice a tile: 64 experts of 64 rows, 2048 x 1408, 108 us, 101 so.)
__device__ __forceinline__ int64_t stream_rows(const SlotRows& at, int e, int64_t& first) {
  typedef const __attribute__((address_space(4))) int32_t fixed;
  first = 0;
  if (at.offsets == nullptr) return at.rows;
  fixed* p = (fixed*)(uintptr_t)(at.offsets + e);
  first = bounded(p[0], at.rows);
  return max((int64_t)0, bounded(p[1], at.rows) - first);
}
template <class T, int TI, int TJ, int SLOTS>
struct DwStream {
  typedef kn::Tile<T, true, TI, TJ, SLOTS> G;
  static constexpr int kStreamers = 256 * G::kWaves;
  struct Shared {
    typename G::Ring ring;
    struct Stage {
      char b[4 * 16 * 32 * TJ];
    } stage;
    uint16_t order[kMaxExperts];  // experts by falling rows
  };

  struct Tiles {
    const ExpertGradArgs& a;
    const Shared& sh;
    uint32_t mt, ntl, share, at, expert;
    int64_t m0, n0;

    __device__ __forceinline__ bool next(kn::Side& P, kn::Side& Q, int64_t& k) {
      for (;;) {
        const uint32_t which = at / share;
        if (which >= (uint32_t)a.at.experts) return false;
        const uint32_t tile = (blockIdx.x & 7) * share + (at - which * share);
        at += kStreamers / 8;
        if (tile >= mt * ntl) continue;
        expert = __builtin_amdgcn_readfirstlane((int)sh.order[which]);
        uint32_t ti, tj;
        tile_at(tile, mt, ntl, ti, tj);
        m0 = (int64_t)ti * G::BM;
        n0 = (int64_t)tj * G::BN;
        int64_t row0;
        k = stream_rows(a.at, (int)expert, row0);
        P = {(const char*)(a.g + row0 * a.ldg + m0), a.m - m0, (uint32_t)(a.ldg * 2)};
        Q = {(const char*)(a.x + row0 * a.ldx + n0), a.n - n0, (uint32_t)(a.ldx * 2)};
        return true;
      }
    }
  };
};

template <class T, int TI, int TJ, int SLOTS>
__global__ __launch_bounds__(nt::kThreads, (kn::Tile<T, true, TI, TJ, SLOTS>::kWaves)) void k_expert_dw_stream(
    ExpertGradArgs a, uint32_t mt, uint32_t ntl) {
  typedef DwStream<T, TI, TJ, SLOTS> S;
  typedef typename S::G G;
  __shared__ typename S::Shared sh;
  // each expert's place among them: those with more rows, or as many and a lower number, come first
  uint32_t* rows = reinterpret_cast<uint32_t*>(&sh.ring);
  for (int e = threadIdx.x; e < a.at.experts; e += nt::kThreads) {
    int64_t first;
    rows[e] = (uint32_t)expert_rows(a.at, e, first);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.at.experts; e += nt::kThreads) {
    const uint32_t mine = rows[e];
    int place = 0;
    for (int k = 0; k < a.at.experts; ++k) place += rows[k] > mine || (rows[k] == mine && k < e);
    sh.order[place] = (uint16_t)e;
  }
  __syncthreads();
  if (a.db != nullptr) {
    const uint32_t across = (uint32_t)((a.m + 255) / 256);
    for (uint32_t i = blockIdx.x; i < across * (uint32_t)a.at.experts; i += gridDim.x) {
      const uint32_t e = i / across;
      const int64_t col = (int64_t)(i - e * across) * 256 + threadIdx.x;
      int64_t row0;
      const int64_t count = expert_rows(a.at, (int)e, row0);
      if (col < a.m) sum_column(a, e, row0, count, col);
    }
  }
  typename S::Tiles tiles{a, sh, mt, ntl, (mt * ntl + 7) / 8, blockIdx.x >> 3, 0, 0, 0};
  const int e = sums_exponent(a);
  const bool aligned = a.ldo % 8 == 0 && (uintptr_t)a.out % 16 == 0 && a.ldo * 2 <= nt::kMaxRowBytes;
  int wave = wave_here();
  asm volatile("" : "+s"(wave));  // (kept: asked for again it would be read from scratch, behind all copies)
  G::stream(sh.ring, tiles, [&](const typename G::Acc& acc, const typename S::Tiles& t) {
    bf16_t* to = (bf16_t*)a.out + ((int64_t)t.expert * a.m + t.m0) * a.ldo + t.n0;
    const int64_t rows = a.m - t.m0, cols = a.n - t.n0;
    if (aligned && rows >= G::BM && cols >= G::BN)
      store_whole<G>(sh.stage, acc, to, a.ldo, e, wave);
    else
      store_tile<G>(sh.stage, acc, to, a.ldo, rows, cols, e, wave);
  });
}

template <int TI, int TJ, int SLOTS>
hipError_t dx_tiles(const ExpertGradArgs& a, int splits, hipStream_t s) {
  const int64_t cols = (a.n + 32 * TJ - 1) / (32 * TJ), grid = grid_for(a.at, 32 * TI, cols * splits);
  if (grid > kMaxGrid) return hipErrorInvalidValue;
  hipLaunchKernelGGL((k_expert_dx<TI, TJ, SLOTS>), dim3((uint32_t)grid), dim3(nt::kThreads), 0, s, a, (uint32_t)cols,
                     (uint32_t)splits);
  return hipGetLastError();
}

template <class T, int TI, int TJ, int SLOTS>
hipError_t dw_stream(const ExpertGradArgs& a, hipStream_t s) {
  typedef DwStream<T, TI, TJ, SLOTS> S;
  const int64_t mt = (a.m + 32 * TI - 1) / (32 * TI), ntl = (a.n + 32 * TJ - 1) / (32 * TJ);
  if ((mt * ntl + 7) / 8 * a.at.experts > kMaxGrid) return hipErrorInvalidValue;
  hipLaunchKernelGGL((k_expert_dw_stream<T, TI, TJ, SLOTS>), dim3(S::kStreamers), dim3(nt::kThreads), 0, s, a, (uint32_t)mt,
                     (uint32_t)ntl);
  return hipGetLastError();
}

template <class T, int TI, int TJ, int SLOTS>
hipError_t dw_tiles(const ExpertGradArgs& a, int splits, hipStream_t s) {
  const int64_t mt = (a.m + 32 * TI - 1) / (32 * TI), ntl = (a.n + 32 * TJ - 1) / (32 * TJ);
  const int64_t grid = (mt * ntl * splits + 7) / 8 * 8 * a.at.experts;
  if (grid > kMaxGrid) return hipErrorInvalidValue;
  hipLaunchKernelGGL((k_expert_dw<T, TI, TJ, SLOTS>), dim3((uint32_t)grid), dim3(nt::kThreads), 0, s, a, (uint32_t)mt,
                     (uint32_t)ntl, (uint32_t)splits);
  return hipGetLastError();
}

// Rows of whole 16-byte pieces (zeros, or nothing that is stored, beyond cols).
bool laid_ok(const void* p, int64_t ld, int64_t cols) {
  return (uintptr_t)p % 16 == 0 && ld % 8 == 0 && ld >= laid_ld(cols) && ld * 2 <= nt::kMaxRowBytes;
}

bool dx_ok(const ExpertGradArgs& a, const ExpertPlan& p) {
  return fits(a.at) && a.n > 0 && a.m > 0 && laid_ok(a.g, a.ldg, a.m) && laid_ok(a.w, a.ldw, a.n) && p.splits >= 1 &&
         (p.splits == 1 || a.out_f32);
}
bool dw_ok(const ExpertGradArgs& a, const ExpertPlan& p) {
  return fits(a.at) && a.n > 0 && a.m > 0 && laid_ok(a.g, a.ldg, a.m) && laid_ok(a.x, a.ldx, a.n) && p.splits >= 1 &&
         (p.splits == 1 || a.out_f32) && (a.db == nullptr || a.parts != nullptr) && (!a.f16 || a.inverse != nullptr);
}

}  // namespace

// The fastest tiles by the model of their times that linear_plan has (us: per pair of k
// with a compute unit to itself and with all busy, and around them), for products of
// row_tiles(bm) x cols outputs, k of `pairs`.  How many tiles there are hangs on how the
// rows split: unless that is sure, rounds are not counted whole, but half of one more.
// longest: the pairs of the tile with most of them.  split: k may be cut, for a launch more and
// the partial sums' traffic (4 bytes of `outputs` each).
struct TileForm {
  int ti, tj, slots, wgs;
  double pair, loaded, ends;
};
template <class RowTiles>
ExpertPlan best_tiles(std::initializer_list<TileForm> forms, RowTiles row_tiles, int64_t cols, int64_t pairs, int64_t longest,
                      bool sure, bool split, double outputs) {
  ExpertPlan best{0, 0, 4, 4, 2, 1};
  double least = 1e300;
  for (const TileForm& f : forms) {
    const double tiles = row_tiles(32 * f.ti) * (double)((cols + 32 * f.tj - 1) / (32 * f.tj));
    for (int s : {1, 2, 4, 8, 16}) {
      if (s > 1 && (!split || s * 4 > pairs || tiles * s > 768)) break;
      const double wgs = tiles * s, full = 256.0 * f.wgs;
      const double rounds = sure ? ceil(wgs / full) : std::max(1.0, wgs / full + 0.5);
      double us = rounds * (f.ends + (double)((pairs + s - 1) / s) * (wgs > 256 ? f.loaded : f.pair));
      us = std::max(us, f.ends + (double)((longest + s - 1) / s) * f.pair);
      if (s > 1) us += 5.0 + 8.0 * s * outputs / 4e6;
      if (us < least) {
        least = us;
        best = {0, 0, f.ti, f.tj, f.slots, s};
      }
    }
  }
  return best;
}

ExpertPlan rows_plan(int64_t rows, int experts, int64_t k, int64_t cols, bool split) {
  const double active = (double)std::min<int64_t>(experts, rows);
  // an expert's last tile is half full
  auto row_tiles = [&](int bm) { return experts == 1 ? (double)((rows + bm - 1) / bm) : (double)rows / bm + 0.5 * active; };
  const int64_t pairs = (k + kn::kK - 1) / kn::kK;
  return best_tiles({{8, 8, 2, 1, 1.36, 1.36, 13.0},
                     {6, 8, 2, 1, 1.09, 1.09, 10.0},
                     {4, 8, 3, 1, 0.79, 0.79, 8.0},
                     {4, 4, 2, 2, 0.53, 0.90, 6.0},
                     {2, 4, 3, 2, 0.27, 0.53, 3.5}},
                    row_tiles, cols, pairs, pairs, experts == 1, split, (double)rows * (double)cols);
}

// The few-row form's 16 outputs a workgroup read x anew each time, and start for little where k is short; tiles
// take as long for one row of an expert as for 64, and read W packed where it does not lie in whole 16 bytes.
// us, few-row form and tiles: 4096 -> 2048, 8 experts of one row 33 and 39, of 12 rows 38 and 40, of 48 rows 75 and 42; 64
// experts of one row 189 and 176, of 48 rows 536 and 187.  2048 -> 1408, 24 experts of 8 rows 35 and 43, 64 of 4 rows 67
// and 83, of 12 rows 89 and 83.  1024 -> 1024, 24 of one row 14 and 14, 64 of one 33 and 26.  256 -> 2048, 24 of one
// row 12 and 10, 128 of one 73 and 38.  Packed, 4095 -> 2048: 8 experts of 12 rows 72 and 86, of 24 rows 97 and 86; 64 of 12
// rows 628 and 754, of 24 rows 878 and 766; 1001 -> 777: 8 of 24 rows 16 and 23, 64 of 24 rows 75 and 56.
// 16-row tiles of it a workgroup, 2 experts, 4096 -> 2048: 16 rows by one 12.1 us, by two 12.0; 24 rows by one 18.4, by
// two 14.7 and by four 14.7; 48 rows by two 25.6, by four 20.9.
ExpertPlan expert_plan(int64_t rows, int experts, int64_t n, int64_t m, bool w_lies) {
  const int64_t active = std::min<int64_t>(experts, rows), each = (rows + active - 1) / active;
  const bool little = rows * m <= (int64_t(1) << 18);
  if (each <= 48 && (w_lies ? little && n > 512 : little || each <= 12)) {
    ExpertPlan p{};
    p.nt = each <= 12 ? 1 : each <= 24 ? 2 : 4;
    const int64_t groups = active * ((m + 15) / 16), steps = (n * 2 + 127) / 128;
    p.waves = 4;
    while (p.waves < 16 && groups * p.waves < 2048 && steps >= 8 * p.waves) p.waves *= 2;
    return p;
  }
  return rows_plan(rows, experts, n, m, false);
}

ExpertPlan expert_dx_plan(int64_t rows, int experts, int64_t n, int64_t m) {
  return rows_plan(rows, experts, m, n, true);
}

ExpertPlan expert_dw_plan(int64_t rows, int experts, int64_t n, int64_t m) {
  const int64_t each = std::max<int64_t>(1, rows / std::min<int64_t>(experts, rows));
  auto row_tiles = [&](int bm) { return (double)experts * (double)((m + bm - 1) / bm); };
  // (the fullest expert of a batch has some three times the mean)
  const int64_t pairs = (each + kn::kK - 1) / kn::kK, longest = experts == 1 ? pairs : 3 * pairs;
  return best_tiles({{8, 8, 2, 1, 1.36, 1.36, 10.5}, {4, 4, 2, 2, 0.53, 0.90, each <= 128 ? 4.0 : 6.0}, {2, 4, 3, 2, 0.27, 0.53, 3.5}},
                    row_tiles, n, pairs, longest, true, true, (double)experts * (double)m * (double)n);
}

hipError_t launch_expert_linear(const ExpertArgs& a, const ExpertPlan& p, hipStream_t s) {
  const LinearArgs& l = a.lin;
  if (!fits(a.at) || a.at.order == nullptr || l.n <= 0 || l.m <= 0 || l.n * 2 > nt::kMaxRowBytes) return hipErrorInvalidValue;
  if (p.nt == 0 && (!tile_rows_ok(l.x, l.ldx, l.n, 2) || !tile_rows_ok(l.w, l.ldw, l.n, 2) ||
                    (a.gather && ((a.at.tokens - 1) * l.ldx + l.n) * 2 > (int64_t)nt::kOutside)))
    return hipErrorInvalidValue;
  if (p.nt == 0 && p.splits != 1) return hipErrorInvalidValue;
#define FF_SKINNY(NT, W) \
  if (p.nt == NT && p.waves == W) return expert_skinny<NT, 1, W>(a, s);
  FF_SKINNY(1, 4) FF_SKINNY(1, 8) FF_SKINNY(1, 16) FF_SKINNY(2, 4) FF_SKINNY(2, 8) FF_SKINNY(2, 16) FF_SKINNY(4, 4)
  FF_SKINNY(4, 8) FF_SKINNY(4, 16)
#undef FF_SKINNY
#define FF_TILE(I, J, S) \
  if (p.nt == 0 && p.ti == I && p.tj == J && p.slots == S) return expert_tiles<I, J, S>(a, s);
  FF_TILE(8, 8, 2) FF_TILE(6, 8, 2) FF_TILE(4, 8, 3) FF_TILE(4, 4, 2) FF_TILE(2, 4, 3)
#undef FF_TILE
  return hipErrorInvalidValue;
}

hipError_t launch_combine(const CombineArgs& a, hipStream_t s) {
  if (!fits(a.at) || (a.at.place == nullptr && (!a.f32 || a.at.top != 1)) || a.cols <= 0 || (a.f32 && a.parts < 1))
    return hipErrorInvalidValue;
  const uint32_t per_row = (uint32_t)((a.cols + 7) / 8);
  const int64_t total = a.at.tokens * per_row;
  const dim3 grid((uint32_t)std::min<int64_t>((total + 255) / 256, 1 << 20));
  if (a.f32)
    hipLaunchKernelGGL(k_combine<true>, grid, dim3(256), 0, s, a, per_row, total);
  else
    hipLaunchKernelGGL(k_combine<false>, grid, dim3(256), 0, s, a, per_row, total);
  return hipGetLastError();
}

hipError_t launch_combine_grad(const CombineGradArgs& a, hipStream_t s) {
  if (!fits(a.at) || a.at.place == nullptr || a.at.order == nullptr || a.at.weights == nullptr || a.cols <= 0) return hipErrorInvalidValue;
  hipLaunchKernelGGL(k_combine_grad, dim3((uint32_t)((a.at.rows + 3) / 4)), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_rows(const RowsArgs* jobs, int count, hipStream_t s) {
  if (count < 1 || count > 3) return hipErrorInvalidValue;
  RowsJobs q{};
  int64_t total = 0, numbers = 0;
  for (int k = 0; k < count; ++k) {
    const RowsArgs& a = jobs[k];
    // (rows that are no slots, those of all experts' weights, may be more than slots are)
    const bool plain = a.at.offsets == nullptr && !a.gather && a.parts == nullptr && a.at.rows > 0 && a.at.rows <= (int64_t(1) << 30);
    if ((!plain && !fits(a.at)) || (a.gather && a.at.order == nullptr) || a.cols <= 0 || a.cols > (int64_t(1) << 24)) return hipErrorInvalidValue;
    if ((uintptr_t)a.laid % 16 != 0 || (uintptr_t)a.scaled % 16 != 0 || (a.scaled != nullptr && a.peaks == nullptr))
      return hipErrorInvalidValue;
    if ((a.scaled != nullptr && a.inverse == nullptr) || (a.parts != nullptr && (k != 0 || (uintptr_t)a.parts % 16 != 0)))
      return hipErrorInvalidValue;
    const int64_t per_row = (a.cols + 7) / 8;
    numbers += a.at.rows * a.cols;
    if (a.parts != nullptr) {
      q.part_rows = part_rows(a.at.rows, a.cols);
      int64_t across = 64;  // as k_rows has it
      while (across > 2 && across / 2 >= per_row) across /= 2;
      total += grid_for(a.at, q.part_rows, (per_row + across - 1) / across);
      if (total > kMaxGrid) return hipErrorInvalidValue;
    } else {
      total += std::min<int64_t>((a.at.rows * per_row + 511) / 512, 8192);
    }
    q.job[k] = a;
    q.end[k] = (uint32_t)total;
  }
  for (int k = count; k < 3; ++k) q.end[k] = (uint32_t)total;
  // Few numbers are bound by latency, many by memory, which more waves keep busy.  dW from checkpoints with the activation
  // decided once and not: 1021 x 777 and x 1000 32.5 and 34.3 us, 2048 x 2048 and x 1024 51 and 59, 8192 x 2048 twice 135 and
  // 140, 4096 x 11008 and x 4096 443 and 439; gradients of 64 experts 777 x 1001, whose weights are laid out, 105 and 93
  if (numbers <= (int64_t(1) << 25))
    hipLaunchKernelGGL(k_rows<true>, dim3((uint32_t)total), dim3(256), 0, s, q);
  else
    hipLaunchKernelGGL(k_rows<false>, dim3((uint32_t)total), dim3(256), 0, s, q);
  return hipGetLastError();
}

hipError_t launch_peaks(const RowsArgs& g, uint32_t* g_peaks, const RowsArgs& scales, uint32_t* x_peaks, hipStream_t s) {
  const PeaksJobs q{{g, scales}, {g_peaks, x_peaks}};
  for (int k = 0; k < 2; ++k) {
    const RowsArgs& a = q.job[k];
    if (!fits(a.at) || (a.gather && a.at.order == nullptr) || a.cols <= 0 || a.cols > (int64_t(1) << 24) || a.src == nullptr ||
        q.peaks[k] == nullptr || (uintptr_t)q.peaks[k] % 16 != 0)
      return hipErrorInvalidValue;
  }
  hipLaunchKernelGGL(k_peaks, dim3(2 * kPeaks), dim3(256), 0, s, q);
  return hipGetLastError();
}

hipError_t launch_expert_dx(const ExpertGradArgs& a, const ExpertPlan& p, hipStream_t s) {
  if (!dx_ok(a, p)) return hipErrorInvalidValue;
#define FF_TILE(I, J, S) \
  if (p.ti == I && p.tj == J && p.slots == S) return dx_tiles<I, J, S>(a, p.splits, s);
  FF_TILE(8, 8, 2) FF_TILE(6, 8, 2) FF_TILE(4, 8, 3) FF_TILE(4, 4, 2) FF_TILE(2, 4, 3)
#undef FF_TILE
  return hipErrorInvalidValue;
}

hipError_t launch_expert_dw(const ExpertGradArgs& a, const ExpertPlan& p, hipStream_t s) {
  if (!dw_ok(a, p)) return hipErrorInvalidValue;
#define FF_STREAM(I, J, S)                                                                                   \
  if (p.ti == I && p.tj == J && p.slots == S && p.splits == 1 && !a.out_f32)                                 \
    return a.f16 ? dw_stream<nt::F16, I, J, S>(a, s) : dw_stream<nt::Bf16, I, J, S>(a, s);
  FF_STREAM(8, 8, 2)
  // (with more pairs the two workgroups of a unit hide each other's ends as well: in a stream and without, 64 experts of
  // 128 rows, 2048 x 1408, 147 and 162 us, of 256 rows 232 and 270, of 512 rows 380 and 401; 8 experts of 1024 rows
  // 79.7 and 79.0, of 4096 rows 294 and 290; one of 4096 rows, 2048 x 2048, 71 and 67)
  if (a.at.rows <= 512 * (int64_t)a.at.experts) FF_STREAM(4, 4, 2)
#undef FF_STREAM
#define FF_TILE(I, J, S)                       \
  if (p.ti == I && p.tj == J && p.slots == S)  \
    return a.f16 ? dw_tiles<nt::F16, I, J, S>(a, p.splits, s) : dw_tiles<nt::Bf16, I, J, S>(a, p.splits, s);
  FF_TILE(8, 8, 2) FF_TILE(4, 4, 2) FF_TILE(2, 4, 3)
#undef FF_TILE
  return hipErrorInvalidValue;
}

bool expert_both(const ExpertPlan& dx, const ExpertPlan& dw) { return dx.ti == 2 && dw.ti == 2; }

hipError_t launch_expert_both(const ExpertGradArgs& x, const ExpertPlan& px, const ExpertGradArgs& w, const ExpertPlan& pw,
                              hipStream_t s) {
  if (!dx_ok(x, px) || !dw_ok(w, pw) || !expert_both(px, pw)) return hipErrorInvalidValue;
  const int64_t cols = (x.n + 127) / 128, first = (grid_for(x.at, 64, cols * px.splits) + 7) / 8 * 8;
  const int64_t mt = (w.m + 63) / 64, ntl = (w.n + 127) / 128, grid = first + (mt * ntl * pw.splits + 7) / 8 * 8 * w.at.experts;
  if (grid > kMaxGrid) return hipErrorInvalidValue;
  if (w.f16)
    hipLaunchKernelGGL((k_expert_both<nt::F16, 2, 4, 3>), dim3((uint32_t)grid), dim3(nt::kThreads), 0, s, x, (uint32_t)cols,
                       (uint32_t)px.splits, (uint32_t)first, w, (uint32_t)mt, (uint32_t)ntl, (uint32_t)pw.splits);
  else
    hipLaunchKernelGGL((k_expert_both<nt::Bf16, 2, 4, 3>), dim3((uint32_t)grid), dim3(nt::kThreads), 0, s, x, (uint32_t)cols,
                       (uint32_t)px.splits, (uint32_t)first, w, (uint32_t)mt, (uint32_t)ntl, (uint32_t)pw.splits);
  return hipGetLastError();
}

hipError_t launch_expert_db(const ExpertGradArgs& a, hipStream_t s) {
  if (!fits(a.at) || a.m <= 0 || a.parts == nullptr || a.db == nullptr) return hipErrorInvalidValue;
  hipLaunchKernelGGL(k_expert_db, dim3((uint32_t)((a.m + 255) / 256), (uint32_t)a.at.experts), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace ff
