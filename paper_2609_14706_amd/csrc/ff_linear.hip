// Linear layers with bias, activation and residual in the product's epilogue:
//   y_ti = act(s_t b_i sum_j x_tj w_ij + bias_i) + r_ti
// for bf16 (s = b = 1) and for 8-bit rows and codes (V = beta alpha^T (.) Z
// with alpha folded into the rows: s the rows' scales, b = beta), whose
// integer sums are exact.
//
// Many tokens are bound by the matrix cores: tiles of 256 x 256 down to 64 x 128
// (ff_tile_nt.hpp), tiles that run together on an XCD sharing operand rows in
// its L2, k split and joined by a second kernel where tiles are few.  Few
// tokens (up to 64) are bound by reading w once: k_skinny gives every wave 16
// output rows' share of k straight from memory to the matrix cores, with no
// LDS between, and joins the waves' sums at the end.
#include <math.h>

#include <algorithm>
#include <type_traits>
#include <utility>

#include "ff_layer_kernels.hpp"
#include "ff_linear_tile.hpp"
#include "ff_tile_nt.hpp"
#include "ff_vec.hpp"

namespace ff {
namespace {

template <class T, int TI, int TJ, int SLOTS>
__global__ __launch_bounds__(nt::kThreads, (LinearTile<T, TI, TJ, SLOTS>::kWaves)) void k_tile(
    LinearArgs a, uint32_t mt, uint32_t ntl, uint32_t splits, typename Scalar<T>::type* P) {
  typedef LinearTile<T, TI, TJ, SLOTS> L;
  __shared__ typename L::Shared all;
  const uint32_t tiles = mt * ntl;
  const uint32_t w = xcd_remap(blockIdx.x, gridDim.x);
  const uint32_t z = w / tiles;
  uint32_t ti, tj;
  tile_at(w - z * tiles, mt, ntl, ti, tj);
  L::template run<false>(all, a, (int64_t)ti * L::G::BM, (int64_t)tj * L::G::BN, z, splits, P, nullptr, 1, 0);
}

// Sum of the splits' partial sums, in their order, and the epilogue: four
// outputs a thread.
template <class S>
__global__ __launch_bounds__(256) void k_join(LinearArgs a, const S* P, int splits) {
  const int64_t per_row = (a.m + 3) / 4, total = a.tokens * per_row;
  for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < total; id += (int64_t)gridDim.x * 256) {
    const int64_t t = id / per_row, i = (id - t * per_row) * 4;
    const int count = (int)min((int64_t)4, a.m - i);
    S v[4] = {0, 0, 0, 0};
    for (int z = 0; z < splits; ++z) {
      const S* p = P + ((int64_t)z * a.tokens + t) * a.m + i;
      S w[4] = {0, 0, 0, 0};
      if (count == 4) {
        __builtin_memcpy(w, p, sizeof w);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (k < count) w[k] = p[k];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = add(v[k], w[k]);
    }
    float f[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) f[k] = sum_f32(v[k]);
    finish<4>(a, t, i, f, count);
  }
}

template <class T, int NT, int RW, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_skinny(LinearArgs a) {
  __shared__ SkinnySums<T, NT, RW, WAVES> sh;
  skinny_run<T, NT, RW, WAVES, false>(sh, a, (int64_t)blockIdx.x * (16 * RW), nullptr, 1, 0);
}

template <int EB>
__global__ __launch_bounds__(256) void k_pack_rows(const char* src, int64_t ld, int64_t rows, int64_t n, char* dst,
                                                   int64_t ldd) {
  const int64_t chunks = ldd * EB / 16, total = rows * chunks;
  for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < total; id += (int64_t)gridDim.x * 256) {
    const int64_t r = id / chunks, c = id - r * chunks;
    const u32x4 v = row_bytes<EB>(src + r * ld * EB, (int)(c * 16), (int)(n * EB));
    *reinterpret_cast<u32x4*>(dst + r * ldd * EB + c * 16) = v;
  }
}

template <class E>
__global__ __launch_bounds__(256) void k_zero(E* dst, int64_t ld, int64_t rows, int64_t cols) {
  const int64_t total = rows * cols;
  for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < total; id += (int64_t)gridDim.x * 256)
    dst[id / cols * ld + id % cols] = E(0);
}

// 64 x 64 elements through LDS (rows of 33 words: a transposed read of pairs
// spreads over the banks); 256 threads, 16 elements each way a thread.
struct __align__(16) Turn {
  bf16_t e[64][66];
};

// Up to three jobs in one launch, each a range of workgroups.
struct TurnJobs {
  ActGradArgs job[3];
  uint32_t end[3], gx[3];  // first workgroup after the job, its 64-column blocks
};

__global__ __launch_bounds__(256) void k_turn(TurnJobs jobs) {
  __shared__ Turn sm;
  __shared__ float sums[4][64];
  const int which = (blockIdx.x >= jobs.end[0]) + (blockIdx.x >= jobs.end[1]);
  const ActGradArgs& a = jobs.job[which];
  const uint32_t w = blockIdx.x - (which > 0 ? jobs.end[which - 1] : 0), by = w / jobs.gx[which];
  const int64_t r0 = (int64_t)by * 64, c0 = (int64_t)(w - by * jobs.gx[which]) * 64;
  const int tid = threadIdx.x;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = (tid >> 3) + 32 * h, c = (tid & 7) * 8;
    const int64_t row = r0 + r, col = c0 + c;
    const int count = row < a.rows ? (int)min((int64_t)8, max((int64_t)0, a.cols - col)) : 0;
    Vec<bf16_t> v;
    v.w = u32x4{0, 0, 0, 0};
    if (count > 0) v = load_row(a.dy + row * a.lddy + col, count);
    if (a.z != nullptr && count > 0) {
      const Vec<bf16_t> z = load_row(a.z + row * a.ldz + col, count);
      float f[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] = v.get(k) * act_slope(z.get(k), a.act);
      v.set(f);
    }
    if (a.g != nullptr && count > 0) store_row(a.g + row * a.ldg + col, v, count);
#pragma unroll
    for (int k = 0; k < 8; ++k) sm.e[r][c + k] = k < count ? v.bits(k) : (bf16_t)0;
  }
  __syncthreads();
  if (a.part != nullptr) {
    const int c = tid & 63, g = tid >> 6;
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; ++k) s += bf16_to_f32(sm.e[g * 16 + k][c]);
    sums[g][c] = s;
    __syncthreads();
    if (g == 0 && c0 + c < a.cols)
      a.part[(int64_t)by * a.cols + c0 + c] = s + sums[1][c] + sums[2][c] + sums[3][c];
  }
  if (a.gt == nullptr) return;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int c = (tid >> 3) + 32 * h, r = (tid & 7) * 8;
    if (c0 + c >= a.cols || r0 + r >= a.ldgt) continue;
    Vec<bf16_t> v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v.w[k] = (uint32_t)sm.e[r + 2 * k][c] | ((uint32_t)sm.e[r + 2 * k + 1][c] << 16);
    store_row(a.gt + (c0 + c) * a.ldgt + r0 + r, v, 8);  // ldgt is a multiple of 8
  }
}

template <class T, int TI, int TJ, int SLOTS>
hipError_t tiles(const LinearArgs& a, const LinearPlan& p, void* partial, hipStream_t s) {
  typedef nt::Tile<T, TI, TJ, SLOTS> G;
  const int64_t mt = (a.tokens + G::BM - 1) / G::BM, ntl = (a.m + G::BN - 1) / G::BN;
  const int64_t wgs = mt * ntl * p.splits;
  if (wgs > 0x7fffffff || (p.splits > 1 && partial == nullptr)) return hipErrorInvalidValue;
  typedef typename Scalar<T>::type S;
  hipLaunchKernelGGL((k_tile<T, TI, TJ, SLOTS>), dim3((uint32_t)wgs), dim3(nt::kThreads), 0, s, a, (uint32_t)mt,
                     (uint32_t)ntl, (uint32_t)p.splits, p.splits > 1 ? (S*)partial : nullptr);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  const int64_t blocks = std::min<int64_t>((a.tokens * ((a.m + 3) / 4) + 255) / 256, 4096);
  hipLaunchKernelGGL(k_join<S>, dim3((uint32_t)blocks), dim3(256), 0, s, a, (const S*)partial, p.splits);
  return hipGetLastError();
}

// Waves that a form of the few-token kernel is ever given: two output tiles are for
// 256 workgroups and more, with which eight waves do, and for more than 32 tokens
// only a short k is taken there at all.
constexpr int most_waves(int nt, int rw) { return rw == 1 ? 16 : nt == 2 ? 8 : 4; }

template <class T, int NT, int RW>
hipError_t skinny_waves(const LinearArgs& a, int waves, hipStream_t s) {
  const dim3 grid((uint32_t)((a.m + 16 * RW - 1) / (16 * RW)));
  if (waves == 4) {
    hipLaunchKernelGGL((k_skinny<T, NT, RW, 4>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
  }
  if constexpr (most_waves(NT, RW) >= 8)
    if (waves == 8) {
      hipLaunchKernelGGL((k_skinny<T, NT, RW, 8>), grid, dim3(512), 0, s, a);
      return hipGetLastError();
    }
  if constexpr (most_waves(NT, RW) >= 16)
    if (waves == 16) {
      hipLaunchKernelGGL((k_skinny<T, NT, RW, 16>), grid, dim3(1024), 0, s, a);
      return hipGetLastError();
    }
  return hipErrorInvalidValue;
}

template <class T>
hipError_t linear_for(const LinearArgs& a, const LinearPlan& p, void* partial, hipStream_t s) {
  if (p.skinny) {
    const SkinnyPlan k = skinny_plan(a.tokens, a.n, a.m, T::kBytes);
    if (k.nt == 1) return skinny_waves<T, 1, 1>(a, k.waves, s);
    if (k.nt == 2) return k.rw == 2 ? skinny_waves<T, 2, 2>(a, k.waves, s) : skinny_waves<T, 2, 1>(a, k.waves, s);
    return k.rw == 2 ? skinny_waves<T, 4, 2>(a, k.waves, s) : skinny_waves<T, 4, 1>(a, k.waves, s);
  }
#define FF_TILE(I, J, S) \
  if (p.ti == I && p.tj == J && p.slots == S) return tiles<T, I, J, S>(a, p, partial, s);
  FF_TILE(8, 8, 2) FF_TILE(6, 8, 2) FF_TILE(4, 8, 3) FF_TILE(4, 6, 3) FF_TILE(4, 4, 2) FF_TILE(4, 4, 4) FF_TILE(2, 4, 3)
#undef FF_TILE
  return hipErrorInvalidValue;
}

}  // namespace

LinearPlan linear_plan(int64_t tokens, int64_t n, int64_t m, int elem_bytes) {
  // The fastest of the forms below by a model of their times (us), fitted to
  // sweeps of both types from 1 to 4096 tokens and 300 to 28672 wide.  Per pair
  // of k a workgroup takes `pair` (the latency of its copies, or its products)
  // while it has a compute unit to itself and `loaded` when all are busy; where
  // w goes by once (one row of tiles) memory's latency, 0.47, at least, and the
  // workgroups' share of reading it at 6.6 TB/s.  `ends` is its start and
  // epilogue.  A join of splits costs a launch and the partial sums' traffic.
  struct Form {
    int ti, tj, slots, wgs;
    double pair, loaded, ends;
  };
  static const Form forms[] = {{8, 8, 2, 1, 1.36, 1.36, 13.0}, {6, 8, 2, 1, 1.09, 1.09, 10.0}, {4, 8, 3, 1, 0.79, 0.79, 8.0},
                               {4, 6, 3, 1, 0.61, 0.61, 7.0},  {4, 4, 2, 2, 0.53, 0.85, 6.5},  {4, 4, 4, 1, 0.42, 0.53, 5.0},
                               {2, 4, 3, 2, 0.27, 0.53, 3.0}};
  const int64_t pairs = (n * elem_bytes + nt::kPair - 1) / nt::kPair;
  LinearPlan best{false, 8, 8, 2, 1};
  double least = 1e300;
  for (const Form& f : forms) {
    const int64_t rows = (tokens + 32 * f.ti - 1) / (32 * f.ti), tiles = rows * ((m + 32 * f.tj - 1) / (32 * f.tj));
    for (int s : {1, 2, 3, 4, 6, 8, 12, 16}) {
      if (s > 1 && (s * 4 > pairs || tiles * s > 768 || f.ti * f.tj > 16)) break;
      const int64_t wgs = tiles * s, rounds = (wgs + 256 * f.wgs - 1) / (256 * f.wgs);
      double pair = wgs > 256 ? f.loaded : f.pair;
      if (rows == 1)
        pair = std::max({pair, 0.47, (double)std::min<int64_t>(wgs, 256 * f.wgs) * (32 * f.tj * nt::kPair) / 6.6e6});
      double us = (double)rounds * (f.ends + (double)((pairs + s - 1) / s) * pair);
      if (s > 1) us += 5.0 + 8.0 * (double)s * (double)tokens * (double)m / 4e6;
      if (us < least) {
        least = us;
        best = {false, f.ti, f.tj, f.slots, s};
      }
    }
  }
  if (tokens <= 64) {
    // straight from memory: what 16, 32 or 64 tokens a wave leave of its rate
    const double rate = tokens <= 16 ? 4.5e6 : tokens <= 32 ? 3.3e6 : 2.3e6;
    if (2.0 + (double)m * (double)n * elem_bytes / rate < least) return {true, 0, 0, 0, 1};
  }
  return best;
}

SkinnyPlan skinny_plan(int64_t tokens, int64_t n, int64_t m, int elem_bytes) {
  const int nt = tokens <= 16 ? 1 : tokens <= 32 ? 2 : 4, rw = nt > 1 && m >= 8192 ? 2 : 1;
  const int64_t groups = (m + 16 * rw - 1) / (16 * rw), steps = (n * elem_bytes + 127) / 128;
  // enough waves to keep memory busy (8 a compute unit), each with four steps
  // or more
  int waves = 4;
  while (waves < most_waves(nt, rw) && groups * waves < 2048 && steps >= 8 * waves) waves *= 2;
  return {nt, rw, waves};
}

size_t linear_partial_bytes(const LinearPlan& p, int64_t tokens, int64_t m) {
  return p.splits > 1 ? (size_t)p.splits * (size_t)tokens * (size_t)m * 4 : 0;
}

bool tile_rows_ok(const void* p, int64_t ld, int64_t n, int elem_bytes) {
  return (uintptr_t)p % 16 == 0 && ld * elem_bytes % 16 == 0 && n * elem_bytes % 16 == 0 &&
         ld * elem_bytes <= nt::kMaxRowBytes;
}

int64_t packed_ld(int64_t n, int elem_bytes) {
  const int64_t g = nt::kPair / elem_bytes;
  return (n + g - 1) / g * g;
}

hipError_t launch_pack_rows(const void* src, int64_t ld, int64_t rows, int64_t n, int elem_bytes, void* dst,
                            hipStream_t s) {
  if (rows <= 0 || n <= 0 || n * elem_bytes > nt::kMaxRowBytes || (uintptr_t)dst % 16 != 0)
    return hipErrorInvalidValue;
  const int64_t ldd = packed_ld(n, elem_bytes);
  const dim3 grid((uint32_t)std::min<int64_t>((rows * (ldd * elem_bytes / 16) + 255) / 256, 8192));
  if (elem_bytes == 1)
    hipLaunchKernelGGL(k_pack_rows<1>, grid, dim3(256), 0, s, (const char*)src, ld, rows, n, (char*)dst, ldd);
  else if (elem_bytes == 2)
    hipLaunchKernelGGL(k_pack_rows<2>, grid, dim3(256), 0, s, (const char*)src, ld, rows, n, (char*)dst, ldd);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

hipError_t launch_linear(const LinearArgs& a, const LinearPlan& p, int elem_bytes, void* partial, hipStream_t s) {
  if (a.tokens <= 0 || a.n <= 0 || a.m <= 0 || a.n * elem_bytes > nt::kMaxRowBytes) return hipErrorInvalidValue;
  if (p.skinny ? a.tokens > 64
               : !tile_rows_ok(a.x, a.ldx, a.n, elem_bytes) || !tile_rows_ok(a.w, a.ldw, a.n, elem_bytes) ||
                     p.splits < 1)
    return hipErrorInvalidValue;
  if (elem_bytes == 1) return linear_for<nt::I8>(a, p, partial, s);
  if (elem_bytes == 2) return linear_for<nt::Bf16>(a, p, partial, s);
  return hipErrorInvalidValue;
}

hipError_t launch_zero(void* dst, int64_t ld, int64_t rows, int64_t cols, int elem_bytes, hipStream_t s) {
  if (rows <= 0 || cols <= 0) return hipErrorInvalidValue;
  const dim3 grid((uint32_t)std::min<int64_t>((rows * cols + 255) / 256, 4096));
  if (elem_bytes == 2)
    hipLaunchKernelGGL(k_zero<uint16_t>, grid, dim3(256), 0, s, (uint16_t*)dst, ld, rows, cols);
  else if (elem_bytes == 4)
    hipLaunchKernelGGL(k_zero<uint32_t>, grid, dim3(256), 0, s, (uint32_t*)dst, ld, rows, cols);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

int64_t act_grad_parts(int64_t rows) { return (rows + 63) / 64; }

hipError_t launch_act_grad(const ActGradArgs* jobs, int count, hipStream_t s) {
  if (count < 1 || count > 3) return hipErrorInvalidValue;
  TurnJobs q{};
  int64_t total = 0;
  for (int k = 0; k < count; ++k) {
    const ActGradArgs& a = jobs[k];
    const int64_t gx = (a.cols + 63) / 64, gy = (a.rows + 63) / 64;
    if (a.rows <= 0 || a.cols <= 0 || gx * gy > 0x7fffffff ||
        (a.gt != nullptr && (a.ldgt % 8 != 0 || a.ldgt < a.rows || a.ldgt > gy * 64 || (uintptr_t)a.gt % 16 != 0)))
      return hipErrorInvalidValue;
    total += gx * gy;
    if (total > 0x7fffffff) return hipErrorInvalidValue;
    q.job[k] = a;
    q.gx[k] = (uint32_t)gx;
    q.end[k] = (uint32_t)total;
  }
  for (int k = count; k < 3; ++k) q.end[k] = (uint32_t)total;
  hipLaunchKernelGGL(k_turn, dim3((uint32_t)total), dim3(256), 0, s, q);
  return hipGetLastError();
}

}  // namespace ff
