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
// Rows of the batch that are in an expert, and an expert's: their number, and the first.
__device__ __forceinline__ int64_t used_rows(const SlotRows& at) {
  return at.offsets == nullptr ? at.rows : bounded(at.offsets[at.experts], at.rows);
}
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

// The workgroup's tile among row tiles of bm rows and `cols` tile columns; false, with
// `extra` its number among those, for workgroups beyond the last tile.
__device__ __forceinline__ bool find_tile(const SlotRows& at, int bm, uint32_t cols, GroupTile& g, uint32_t& extra,
                                          uint32_t& extras) {
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
  const uint32_t used = (uint32_t)min(total, (uint64_t)gridDim.x);
  if (blockIdx.x >= used) {
    extra = blockIdx.x - used;
    extras = gridDim.x - used;
    return false;
  }
  const uint32_t t = xcd_remap(blockIdx.x, used);
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

// Rows in no expert, `bytes` each (a multiple of E's), are set to zeros.
template <class E>
__device__ __forceinline__ void clear_rows(const SlotRows& at, E* p, int64_t ld, int64_t cols, uint32_t extra,
                                           uint32_t extras) {
  for (int64_t r = used_rows(at) + extra; r < at.rows; r += extras)
    for (int64_t c = threadIdx.x; c < cols; c += blockDim.x) p[r * ld + c] = E(0);
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

template <int TI, int TJ, int SLOTS, bool GATHER>
__global__ __launch_bounds__(nt::kThreads, (LinearTile<nt::Bf16, TI, TJ, SLOTS>::kWaves)) void k_expert_tile(
    ExpertArgs x, uint32_t cols) {
  typedef LinearTile<nt::Bf16, TI, TJ, SLOTS> L;
  __shared__ typename L::Shared all;
  GroupTile g;
  uint32_t extra, extras;
  if (!find_tile(x.at, L::G::BM, cols, g, extra, extras)) {
    clear_outputs(x, extra, extras);
    return;
  }
  const LinearArgs a = args_of(x, g);
  L::template run<GATHER>(all, a, 0, (int64_t)g.col * L::G::BN, 0, 1, nullptr, x.at.order + g.row0, x.at.top,
                          x.at.tokens);
}

template <int NT, int RW, int WAVES, bool GATHER>
__global__ __launch_bounds__(64 * WAVES) void k_expert_skinny(ExpertArgs x, uint32_t cols) {
  __shared__ SkinnySums<nt::Bf16, NT, RW, WAVES> sh;
  GroupTile g;
  uint32_t extra, extras;
  if (!find_tile(x.at, 16 * NT, cols, g, extra, extras)) {
    clear_outputs(x, extra, extras);
    return;
  }
  g.rows = min(g.rows, 16 * NT);
  const LinearArgs a = args_of(x, g);
  skinny_run<nt::Bf16, NT, RW, WAVES, GATHER>(sh, a, (int64_t)g.col * (16 * RW), x.at.order + g.row0, x.at.top,
                                              x.at.tokens);
}

// ---------------------------------------------------------------- combining
// Eight columns a thread; the token's rows one after the other, in fp32.
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

// A wave a row: the row's gradient and its weight's.  The wave of number p also
// clears the weight's gradient of slot p where that is in no row.
__global__ __launch_bounds__(256) void k_combine_grad(CombineGradArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t used = used_rows(a.at);
  for (int64_t p = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); p < a.at.rows; p += (int64_t)gridDim.x * 4) {
    const int32_t place = a.at.place[p];
    if (a.dweights != nullptr && lane == 0 && (place < 0 || place >= a.at.rows)) a.dweights[p] = 0.0f;
    const int32_t slot = p < used ? a.at.order[p] : -1;
    const bool live = slot >= 0 && slot < a.at.rows;
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
      if (lane == 0) a.dweights[slot] = dot;
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

struct PeaksJobs {
  PeaksArgs job[2];
};
template <class E>
__device__ __forceinline__ uint32_t peak_bits(const PeaksArgs& a, int64_t block, int64_t blocks) {
  constexpr int N = Vec<E>::N, U = 4;
  uint32_t big = 0;
  const uint32_t per_row = (uint32_t)((a.cols + N - 1) / N);
  const int64_t total = a.rows * per_row;
  for (int64_t b = block * (256 * U); b < total; b += blocks * (256 * U)) {
    const int64_t r = b / per_row;
    Vec<E> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t c = (uint32_t)(b - r * per_row) + u * 256 + threadIdx.x;
      const int64_t row = r + c / per_row, col = (int64_t)(c % per_row) * N;
      v[u].w = u32x4{0, 0, 0, 0};
      if (row < a.rows) v[u] = load_row((const E*)a.src + row * a.ld + col, a.cols - col);
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
__global__ __launch_bounds__(256) void k_peaks(PeaksJobs jobs) {
  __shared__ uint32_t red[4];
  const PeaksArgs& a = jobs.job[blockIdx.x >= kPeaks];
  const int block = blockIdx.x % kPeaks;
  uint32_t big = a.f32 ? peak_bits<float>(a, block, kPeaks) : peak_bits<bf16_t>(a, block, kPeaks);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) big = max(big, (uint32_t)__shfl_xor((int)big, d));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = big;
  __syncthreads();
  if (threadIdx.x == 0) a.peaks[block] = max(max(red[0], red[1]), max(red[2], red[3]));
}

struct RowsJobs {
  RowsArgs job[3];
  uint32_t end[3];  // first workgroup after the job
};

__global__ __launch_bounds__(256) void k_rows(RowsJobs jobs) {
  __shared__ uint32_t red[4];
  const int which = (blockIdx.x >= jobs.end[0]) + (blockIdx.x >= jobs.end[1]);
  const RowsArgs& a = jobs.job[which];
  const uint32_t first = which > 0 ? jobs.end[which - 1] : 0, blocks = jobs.end[which] - first;
  const uint32_t per_row = (uint32_t)((a.cols + 7) / 8);
  const int64_t total = a.at.rows * per_row;
  float scale = 1.0f;
  const int64_t ldl = (int64_t)per_row * 8;
  if (a.scaled != nullptr) scale = ldexpf(1.0f, peak_exponent(peak_of(a.peaks, red), a.peak_factor));
  const int64_t used = used_rows(a.at);
  constexpr int U = 2;
  for (int64_t b = (int64_t)(blockIdx.x - first) * (256 * U); b < total; b += (int64_t)blocks * (256 * U)) {
    const int64_t r = b / per_row;
    float f[U][8];
    int64_t row[U], col[U];
    int count[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t c = (uint32_t)(b - r * per_row) + u * 256 + threadIdx.x;
      row[u] = r + c / per_row;
      col[u] = (int64_t)(c % per_row) * 8;
      count[u] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) f[u][i] = 0.0f;
      if (row[u] >= a.at.rows) continue;
      const int n = (int)min((int64_t)8, a.cols - col[u]);
      count[u] = n;
      if (row[u] >= used) continue;
      const int64_t from = a.gather ? token_of(a.at, row[u]) : row[u];
      if (from < 0) continue;
      if (a.src_q8.q != nullptr) {
        load_q8(a.src_q8, from, col[u], n, f[u]);
#pragma unroll
        for (int i = 0; i < 8; ++i)  // (a NaN scale)
          if (i >= n) f[u][i] = 0.0f;
      } else if (a.src_f32) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (n > 4 * h) {
            const Vec<float> v = load_row((const float*)a.src + from * a.lds + col[u] + 4 * h, n - 4 * h);
#pragma unroll
            for (int i = 0; i < 4; ++i) f[u][4 * h + i] = v.get(i);
          }
      } else {
        const Vec<bf16_t> v = load_row((const bf16_t*)a.src + from * a.lds + col[u], n);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[u][i] = v.get(i);
      }
      if (a.z_q8.q != nullptr) {
        float z[8];
        load_q8(a.z_q8, row[u], col[u], n, z);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < n) f[u][i] *= act_slope(z[i], a.act);
      } else if (a.z != nullptr) {
        const Vec<bf16_t> z = load_row(a.z + row[u] * a.ldz + col[u], n);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[u][i] *= act_slope(z.get(i), a.act);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (count[u] <= 0) continue;
      Vec<bf16_t> o;
      o.set(f[u]);
      if (a.out != nullptr) store_row(a.out + row[u] * a.ldo + col[u], o, count[u]);
      // (elements beyond the row are zeros here)
      if (a.laid != nullptr) *reinterpret_cast<u32x4*>(a.laid + row[u] * ldl + col[u]) = o.w;
      if (a.scaled != nullptr) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          o.w[q] = (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)(f[u][2 * q] * scale)) |
                   (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)(f[u][2 * q + 1] * scale)) << 16;
        *reinterpret_cast<u32x4*>(a.scaled + row[u] * ldl + col[u]) = o.w;
      }
    }
  }
}

// ------------------------------------------------------------------ gradients
// A tile of C to its rows: `rows` and `cols` from the tile's corner on exist, E is
// bf16_t or float.  Each wave turns its own part over in its quarter of the ring, free by then: a
// lane has four columns of a row, and writes 16 bytes beside its neighbours', whole lines of a
// row at once (8192 tiles of 256 x 256 with 256 rows each: 796 us with the lanes' own 8 bytes).
// 16-byte piece c of row r sits at c ^ (r & 15) of its row: 64 banks for either way.
template <class G, class E>
__device__ __forceinline__ void store_tile(typename G::Ring& ring, const typename G::Acc& acc, E* corner, int64_t ld,
                                           int64_t rows, int64_t cols, float f1, float f2) {
  constexpr int TI = (int)(sizeof(typename G::Acc) / sizeof(f32x4[G::BN / 32])), TJ = G::BN / 32;
  constexpr int kLine = 16 * TJ * (int)sizeof(E), kPieces = kLine / 16, kPer = 16 / (int)sizeof(E);  // of a wave's row
  constexpr int kSwz = kPieces < 16 ? kPieces - 1 : 15;
  // tile rows of 16 a phase
  constexpr int kFit = (int)sizeof(typename G::Ring) / 4 / (16 * kLine), H = kFit >= TI ? TI : kFit >= TI / 2 ? TI / 2 : 1;
  static_assert(kFit >= 1 && TI % H == 0 && (16 * H * kPieces) % 64 == 0, "a wave's part of a phase");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  char* mine = reinterpret_cast<char*>(&ring) + wave * (sizeof(typename G::Ring) / 4);
  const int r0 = (wave >> 1) * 16 * TI, c0 = (wave & 1) * 16 * TJ;
#pragma unroll
  for (int h = 0; h < TI / H; ++h) {
#pragma unroll
    for (int i = 0; i < H; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j) {
        const f32x4 a = acc[h * H + i][j];
        const float f[4] = {a[0] * f1 * f2, a[1] * f1 * f2, a[2] * f1 * f2, a[3] * f1 * f2};
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
#pragma unroll 4
    for (int q = lane; q < 16 * H * kPieces; q += 64) {
      const int r = q / kPieces, c = q % kPieces, row = r0 + h * H * 16 + r, col = c0 + c * kPer;
      const u32x4 v = *reinterpret_cast<const u32x4*>(mine + r * kLine + ((c ^ (r & kSwz)) << 4));
      if (row >= rows) continue;
      Vec<E> o;
      o.w = v;
      store_row(corner + row * ld + col, o, cols - col);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// k in `splits` parts: the workgroups of part z are z-th in each XCD's share of the launch.
template <int TI, int TJ, int SLOTS>
__global__ __launch_bounds__(nt::kThreads, (kn::Tile<nt::Bf16, false, TI, TJ, SLOTS>::kWaves)) void k_expert_dx(
    ExpertGradArgs a, uint32_t cols, uint32_t splits) {
  typedef kn::Tile<nt::Bf16, false, TI, TJ, SLOTS> G;
  __shared__ typename G::Ring ring;
  GroupTile g;
  uint32_t extra, extras;
  if (!find_tile(a.at, G::BM, cols * splits, g, extra, extras)) {
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
  typename G::Acc acc;
  G::zero(acc);
  G::loop(ring, P, Q, k1 - k0, acc);
  if (a.out_f32)
    store_tile<G>(ring, acc, (float*)a.out + z * a.part_stride + g.row0 * a.ldo + n0, a.ldo, g.rows, a.n - n0, 1.0f, 1.0f);
  else
    store_tile<G>(ring, acc, (bf16_t*)a.out + g.row0 * a.ldo + n0, a.ldo, g.rows, a.n - n0, 1.0f, 1.0f);
}

// Sums of BM columns of rows of g from `p` on, `cols` of them there.
template <int BM>
__device__ __forceinline__ void column_sums(const ExpertGradArgs& a, const uint16_t* p, int64_t rows, int64_t cols, float factor,
                                            float* lds, bf16_t* out) {
  constexpr int kAcross = BM / 8, kDown = 256 / kAcross;
  const int c = (threadIdx.x % kAcross) * 8, r0 = threadIdx.x / kAcross;
  float s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) s[i] = 0.0f;
  if (c < cols) {  // (whole pieces: zeros beyond the last column)
    auto add = [&](const u32x4& w) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint16_t b = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
        s[i] += a.f16 ? (float)__builtin_bit_cast(_Float16, b) : bf16_to_f32(b);
      }
    };
    int64_t r = r0;
    constexpr int U = 8;
    for (; r + (U - 1) * kDown < rows; r += U * kDown) {
      u32x4 w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) w[u] = *reinterpret_cast<const u32x4*>(p + (r + u * kDown) * a.ldg + c);
#pragma unroll
      for (int u = 0; u < U; ++u) add(w[u]);
    }
    for (; r < rows; r += kDown) add(*reinterpret_cast<const u32x4*>(p + r * a.ldg + c));
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) lds[r0 * BM + c + i] = s[i];
  __syncthreads();
  if (threadIdx.x < BM && (int64_t)threadIdx.x < cols) {
    float v = 0.0f;
#pragma unroll
    for (int k = 0; k < kDown; ++k) v += lds[k * BM + threadIdx.x];
    out[threadIdx.x] = f32_to_bf16(v * factor);
  }
  __syncthreads();
}

// Every XCD takes an eighth of each expert's tiles: their work is the expert's rows,
// and with whole experts to an XCD the fullest one's kept the others waiting (8 experts of 422 to 2247
// rows, 4096 x 4096: 480 us, 292 so).  The tiles of the first columns sum g's
// columns for db as well, whose rows their XCD's L2 has just read.
template <class T, int TI, int TJ, int SLOTS>
__global__ __launch_bounds__(nt::kThreads, (kn::Tile<T, true, TI, TJ, SLOTS>::kWaves)) void k_expert_dw(
    ExpertGradArgs a, uint32_t mt, uint32_t ntl, uint32_t splits) {
  typedef kn::Tile<T, true, TI, TJ, SLOTS> G;
  __shared__ typename G::Ring ring;
  const uint32_t tiles = mt * ntl * splits, share = (tiles + 7) / 8, local = blockIdx.x >> 3, e = local / share;
  const uint32_t tile = (blockIdx.x & 7) * share + (local - e * share);
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
  float f1 = 1.0f, f2 = 1.0f;
  if (a.f16) {
    uint32_t* red = reinterpret_cast<uint32_t*>(&ring);
    f1 = ldexpf(1.0f, -peak_exponent(peak_of(a.g_peaks, red), a.g_factor));
    f2 = ldexpf(1.0f, -peak_exponent(peak_of(a.x_peaks, red), a.x_factor));
  }
  typename G::Acc acc;
  G::zero(acc);
  if (k1 > k0) G::loop(ring, P, Q, k1 - k0, acc);
  if (a.db != nullptr && tj == 0 && z == 0)
    column_sums<G::BM>(a, a.g + row0 * a.ldg + m0, rows, a.m - m0, f1, reinterpret_cast<float*>(&ring), a.db + (int64_t)e * a.m + m0);
  const int64_t at = ((int64_t)e * a.m + m0) * a.ldo + n0;
  if (a.out_f32)
    store_tile<G>(ring, acc, (float*)a.out + z * a.part_stride + at, a.ldo, a.m - m0, a.n - n0, f1, f2);
  else
    store_tile<G>(ring, acc, (bf16_t*)a.out + at, a.ldo, a.m - m0, a.n - n0, f1, f2);
}

// Column sums of an expert's rows: 128 columns a workgroup, 16 threads of eight columns
// side by side, 16 rows at a time.
__global__ __launch_bounds__(256) void k_expert_db(SlotRows at, const bf16_t* g, int64_t ldg, int64_t m, bf16_t* db) {
  __shared__ float sums[16][128];
  const int e = blockIdx.y, tid = threadIdx.x, c = (tid & 15) * 8, r = tid >> 4;
  const int64_t col = (int64_t)blockIdx.x * 128 + c;
  int64_t row0;
  const int64_t row1 = expert_rows(at, e, row0) + row0;
  const int count = (int)min((int64_t)8, max((int64_t)0, m - col));
  float s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) s[i] = 0.0f;
  if (count > 0) {
#pragma unroll 4
    for (int64_t p = row0 + r; p < row1; p += 16) {
      const Vec<bf16_t> v = load_row(g + p * ldg + col, count);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] += v.get(i);
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) sums[r][c + i] = s[i];
  __syncthreads();
  if (tid < 128 && (int64_t)blockIdx.x * 128 + tid < m) {
    float v = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; ++k) v += sums[k][tid];
    db[(int64_t)e * m + (int64_t)blockIdx.x * 128 + tid] = f32_to_bf16(v);
  }
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

template <int TI, int TJ, int SLOTS>
hipError_t dx_tiles(const ExpertGradArgs& a, int splits, hipStream_t s) {
  const int64_t cols = (a.n + 32 * TJ - 1) / (32 * TJ), grid = grid_for(a.at, 32 * TI, cols * splits);
  if (grid > kMaxGrid) return hipErrorInvalidValue;
  hipLaunchKernelGGL((k_expert_dx<TI, TJ, SLOTS>), dim3((uint32_t)grid), dim3(nt::kThreads), 0, s, a, (uint32_t)cols,
                     (uint32_t)splits);
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

}  // namespace

// The fastest tiles by the model of their times that linear_plan has (us: per pair of k
// with a compute unit to itself and with all busy, and around them), for products of
// row_tiles(bm) x cols outputs, k of `pairs`.  How many tiles there are hangs on how the
// rows split: unless that is sure, rounds are not counted whole, but half of one more.
// split: k may be cut, for a launch more and the partial sums' traffic (4 bytes of `outputs` each).
struct TileForm {
  int ti, tj, slots, wgs;
  double pair, loaded, ends;
};
constexpr TileForm kForms[] = {{8, 8, 2, 1, 1.36, 1.36, 13.0}, {6, 8, 2, 1, 1.09, 1.09, 10.0}, {4, 8, 3, 1, 0.79, 0.79, 8.0},
                               {4, 4, 2, 2, 0.53, 0.85, 6.0},  {2, 4, 3, 2, 0.27, 0.53, 3.5}};
template <class RowTiles>
ExpertPlan best_tiles(std::initializer_list<int> forms, RowTiles row_tiles, int64_t cols, int64_t pairs, bool sure, bool split,
                      double outputs) {
  ExpertPlan best{0, 0, 4, 4, 2, 1};
  double least = 1e300;
  for (int k : forms) {
    const TileForm& f = kForms[k];
    const double tiles = row_tiles(32 * f.ti) * (double)((cols + 32 * f.tj - 1) / (32 * f.tj));
    for (int s : {1, 2, 4, 8, 16}) {
      if (s > 1 && (!split || s * 4 > pairs || tiles * s > 768)) break;
      const double wgs = tiles * s, full = 256.0 * f.wgs;
      const double rounds = sure ? ceil(wgs / full) : std::max(1.0, wgs / full + 0.5);
      double us = rounds * (f.ends + (double)((pairs + s - 1) / s) * (wgs > 256 ? f.loaded : f.pair));
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
  return best_tiles({0, 1, 2, 3, 4}, row_tiles, cols, (k + kn::kK - 1) / kn::kK, experts == 1, split, (double)rows * (double)cols);
}

ExpertPlan expert_plan(int64_t rows, int experts, int64_t n, int64_t m) {
  const int64_t active = std::min<int64_t>(experts, rows), each = (rows + active - 1) / active;
  if (each <= 48) {
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
  return best_tiles({0, 3, 4}, row_tiles, n, (each + kn::kK - 1) / kn::kK, true, true, (double)experts * (double)m * (double)n);
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
  int64_t total = 0;
  for (int k = 0; k < count; ++k) {
    const RowsArgs& a = jobs[k];
    if (!fits(a.at) || (a.gather && a.at.order == nullptr) || a.cols <= 0 || a.cols > (int64_t(1) << 24)) return hipErrorInvalidValue;
    if ((uintptr_t)a.laid % 16 != 0 || (uintptr_t)a.scaled % 16 != 0 || (a.scaled != nullptr && a.peaks == nullptr))
      return hipErrorInvalidValue;
    total += std::min<int64_t>((a.at.rows * ((a.cols + 7) / 8) + 511) / 512, 4096);
    q.job[k] = a;
    q.end[k] = (uint32_t)total;
  }
  for (int k = count; k < 3; ++k) q.end[k] = (uint32_t)total;
  hipLaunchKernelGGL(k_rows, dim3((uint32_t)total), dim3(256), 0, s, q);
  return hipGetLastError();
}

hipError_t launch_peaks(const PeaksArgs (&jobs)[2], hipStream_t s) {
  PeaksJobs q{};
  for (int k = 0; k < 2; ++k) {
    if (jobs[k].rows <= 0 || jobs[k].cols <= 0 || jobs[k].cols > (int64_t(1) << 24) || (uintptr_t)jobs[k].peaks % 16 != 0)
      return hipErrorInvalidValue;
    q.job[k] = jobs[k];
  }
  hipLaunchKernelGGL(k_peaks, dim3(2 * kPeaks), dim3(256), 0, s, q);
  return hipGetLastError();
}

hipError_t launch_expert_dx(const ExpertGradArgs& a, const ExpertPlan& p, hipStream_t s) {
  if (!fits(a.at) || a.n <= 0 || a.m <= 0 || !laid_ok(a.g, a.ldg, a.m) || !laid_ok(a.w, a.ldw, a.n) || p.splits < 1 ||
      (p.splits > 1 && !a.out_f32))
    return hipErrorInvalidValue;
#define FF_TILE(I, J, S) \
  if (p.ti == I && p.tj == J && p.slots == S) return dx_tiles<I, J, S>(a, p.splits, s);
  FF_TILE(8, 8, 2) FF_TILE(6, 8, 2) FF_TILE(4, 8, 3) FF_TILE(4, 4, 2) FF_TILE(2, 4, 3)
#undef FF_TILE
  return hipErrorInvalidValue;
}

hipError_t launch_expert_dw(const ExpertGradArgs& a, const ExpertPlan& p, hipStream_t s) {
  if (!fits(a.at) || a.n <= 0 || a.m <= 0 || !laid_ok(a.g, a.ldg, a.m) || !laid_ok(a.x, a.ldx, a.n) || p.splits < 1 ||
      (p.splits > 1 && !a.out_f32))
    return hipErrorInvalidValue;
#define FF_TILE(I, J, S)                       \
  if (p.ti == I && p.tj == J && p.slots == S)  \
    return a.f16 ? dw_tiles<nt::F16, I, J, S>(a, p.splits, s) : dw_tiles<nt::Bf16, I, J, S>(a, p.splits, s);
  FF_TILE(8, 8, 2) FF_TILE(4, 4, 2) FF_TILE(2, 4, 3)
#undef FF_TILE
  return hipErrorInvalidValue;
}

hipError_t launch_expert_db(const SlotRows& at, const bf16_t* g, int64_t ldg, int64_t m, bf16_t* db, hipStream_t s) {
  if (!fits(at) || m <= 0) return hipErrorInvalidValue;
  hipLaunchKernelGGL(k_expert_db, dim3((uint32_t)((m + 127) / 128), (uint32_t)at.experts), dim3(256), 0, s, at, g, ldg, m, db);
  return hipGetLastError();
}

}  // namespace ff
