// Orthogonalisation of an update by Newton-Schulz products:
//   X = G / (||G||_F + eps);  X <- a X + (b A + c A A) X with A = X X^T,
// an odd polynomial of X's singular values that takes them towards 1 and
// leaves its singular vectors.  X is r x c with r <= c (a tall G is taken
// transposed), so the two symmetric products are of the smaller side.
//
// The products run on the matrix cores in fp16: the operands are bounded (X's
// singular values by the polynomial's range, known on the host), so a fixed
// power of two per operand puts them where fp16 keeps 11 bits, three more than
// bf16 at the same rate.  For bf16 updates one part is enough: every rounding
// of X, A and b A + c A A to fp16 is an eighth of the output's own.  For fp32 updates
// every operand is held as hi + lo (22 bits) and a product is three, hi hi +
// hi lo + lo hi, the k axis running over them one after the other; lo lo, 2^-22
// of the product, is left out.  All sums are fp32.
//
// Each step needs X by rows (A = X X^T) and by columns (B X = B (X^T)^T): the
// last product of a step stores both.  Symmetric products compute the tiles on
// and above the diagonal and store them twice.
#include <math.h>

#include <algorithm>

#include "ff_layer_kernels.hpp"
#include "ff_tile_nt.hpp"

namespace ff {
namespace {

constexpr int kNormParts = 128;  // partial sums of squares per matrix

__device__ __forceinline__ uint16_t f16_bits(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
__device__ __forceinline__ float f16_f32(uint16_t b) { return (float)__builtin_bit_cast(_Float16, b); }

// An r x k operand in one or two fp16 parts (lo: null with one).
struct Parts {
  uint16_t* hi;
  uint16_t* lo;
  int64_t ld, stride;  // row and matrix strides, elements
};

// part[b][p] = sum of squares of share p of matrix b (fp64).
template <class E>
__global__ __launch_bounds__(256) void k_square_sums(const E* g, int64_t ldg, int64_t sg, int64_t m, int64_t n,
                                                     double* part) {
  __shared__ double sh[4];
  const E* G = g + blockIdx.y * sg;
  constexpr int N = Vec<E>::N;
  const int64_t per_row = (n + N - 1) / N, total = m * per_row;
  double s = 0.0;
  for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < total; id += (int64_t)gridDim.x * 256) {
    const int64_t i = id / per_row, j = (id - i * per_row) * N;
    const Vec<E> v = load_row(G + i * ldg + j, n - j);
#pragma unroll
    for (int e = 0; e < N; ++e) s += (double)v.get(e) * (double)v.get(e);
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.y * kNormParts + blockIdx.x] = sh[0] + sh[1] + sh[2] + sh[3];
}

// 1 / (||G||_F + eps) of a matrix from its partial sums, in every thread.
__device__ __forceinline__ double inverse_norm(const double* part, int parts, double eps) {
  __shared__ double total;
  if (threadIdx.x < 64) {
    double s = 0.0;
    for (int k = threadIdx.x; k < parts; k += 64) s += part[k];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
    if (threadIdx.x == 0) total = 1.0 / (sqrt(s) + eps);
  }
  __syncthreads();
  return total;
}

struct __align__(16) TurnF {
  float e[64][65];
};

// The start: `rows` (m x n8) and `cols` (n x m8) get scale G / (||G|| + eps) as
// it is and transposed, zeros up to the next multiple of eight.
template <class E, int PARTS>
__global__ __launch_bounds__(256) void k_start(const E* g, int64_t ldg, int64_t sg, int64_t m, int64_t n,
                                               const double* part, int parts, double eps, float scale, Parts rows,
                                               Parts cols) {
  __shared__ TurnF sm;
  const double inv = inverse_norm(part + blockIdx.z * kNormParts, parts, eps);
  const E* G = g + blockIdx.z * sg;
  const int64_t r0 = (int64_t)blockIdx.y * 64, c0 = (int64_t)blockIdx.x * 64;
  const int64_t n8 = (n + 7) / 8 * 8, m8 = (m + 7) / 8 * 8;
  constexpr int N = Vec<E>::N;
  for (int id = threadIdx.x; id < 64 * (64 / N); id += 256) {
    const int r = id / (64 / N), c = id % (64 / N) * N;
    Vec<E> v;
    v.w = u32x4{0, 0, 0, 0};
    if (r0 + r < m && c0 + c < n) v = load_row(G + (r0 + r) * ldg + c0 + c, n - c0 - c);
#pragma unroll
    for (int e = 0; e < N; ++e) sm.e[r][c + e] = (float)((double)v.get(e) * inv) * scale;
  }
  __syncthreads();
  for (int id = threadIdx.x; id < 64 * 8 * 2; id += 256) {
    const bool turned = id >= 512;
    const int r = (id & 511) >> 3, c = (id & 7) * 8;
    const Parts& o = turned ? cols : rows;
    const int64_t row = (turned ? c0 : r0) + r, col = (turned ? r0 : c0) + c;
    if (row >= (turned ? n : m) || col >= (turned ? m8 : n8)) continue;
    u32x4 hi, lo;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint32_t h = 0, l = 0;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int k = c + 2 * q + e;
        const float x = turned ? sm.e[k][r] : sm.e[r][k];
        const uint16_t b = f16_bits(x);
        h |= (uint32_t)b << (16 * e);
        l |= (uint32_t)f16_bits(x - f16_f32(b)) << (16 * e);
      }
      hi[q] = h;
      lo[q] = l;
    }
    const int64_t at = blockIdx.z * o.stride + row * o.ld + col;
    *reinterpret_cast<u32x4*>(o.hi + at) = hi;
    if (PARTS == 2) *reinterpret_cast<u32x4*>(o.lo + at) = lo;
  }
}

// One product of a step, C = L R^T with L: rows x k, R: cols x k.
//   out = alpha C + beta D, D (nullable) laid out as C, in parts;
// stored by rows (o) and by columns (t), or as the result (user, E).
struct StepArgs {
  int64_t rows, cols, k;  // k a multiple of 8 (the operands' zeros included)
  Parts L, R, D, o, t;
  float alpha, beta;
  void* user;  // the result: element (i, j) at i si + j sj
  int64_t si, sj, su;
  int bf16;
  int mt, ntl;  // tiles
};

// Upper tile `idx` of a T x T grid, column by column: (0,0), (0,1), (1,1), ...
__device__ __forceinline__ void upper_at(uint32_t idx, uint32_t& i, uint32_t& j) {
  uint32_t c = (uint32_t)((sqrtf(8.0f * (float)idx + 1.0f) - 1.0f) * 0.5f);
  while ((c + 1) * (c + 2) / 2 <= idx) ++c;
  while (c * (c + 1) / 2 > idx) --c;
  j = c;
  i = idx - c * (c + 1) / 2;
}

__device__ __forceinline__ void put4(uint16_t* p, const uint16_t (&v)[4]) { __builtin_memcpy(p, v, 8); }

template <int PARTS, int TI, int TJ, bool SYM>
__global__ __launch_bounds__(nt::kThreads, (TI * TJ > 32 ? 1 : 2)) void k_step(StepArgs a) {
  typedef nt::Tile<nt::F16, TI, TJ, 2> G;
  __shared__ typename G::Ring sm;
  const uint32_t w = xcd_remap(blockIdx.x, gridDim.x);
  uint32_t ti, tj;
  if (SYM) {
    upper_at(w, ti, tj);
  } else {
    const uint32_t strip = w / (8 * a.ntl), u = w - strip * 8 * a.ntl, r = min(8u, a.mt - strip * 8);
    ti = strip * 8 + u % r;
    tj = u / r;
  }
  const int64_t i0 = (int64_t)ti * G::BM, j0 = (int64_t)tj * G::BN, z = blockIdx.y;
  const nt::Rows A{nullptr, (int)min((int64_t)G::BM, a.rows - i0), (uint32_t)(a.L.ld * 2)};
  const nt::Rows B{nullptr, (int)min((int64_t)G::BN, a.cols - j0), (uint32_t)(a.R.ld * 2)};
  const int64_t la = z * a.L.stride + i0 * a.L.ld, rb = z * a.R.stride + j0 * a.R.ld;
  const int kbytes = (int)a.k * 2, pairs = (kbytes + nt::kPair - 1) / nt::kPair;
  typename G::Acc acc;
  G::zero(acc);
  // two parts: hi lo, lo hi, then hi hi (the largest last)
  G::loop(
      sm, A, B, 0, PARTS == 2 ? 3 * pairs : pairs,
      [&](int p, const char*& pa, const char*& pb) {
        p = __builtin_amdgcn_readfirstlane(p);
        const int seg = PARTS == 2 ? (p >= pairs) + (p >= 2 * pairs) : 2;
        const int k = (PARTS == 2 ? p - seg * pairs : p) * nt::kPair;
        pa = (const char*)((PARTS == 2 && seg == 1 ? a.L.lo : a.L.hi) + la) + k;
        pb = (const char*)((PARTS == 2 && seg == 0 ? a.R.lo : a.R.hi) + rb) + k;
      },
      [&](int p) {
        const int seg = PARTS == 2 ? (p >= pairs) + (p >= 2 * pairs) : 0;
        return kbytes - (p - seg * pairs) * nt::kPair;
      },
      acc);
  // through LDS as in the linear layers: each lane its own slots
  constexpr int HI = TI < 4 ? TI : 4, V = TJ / 4;
  static_assert(TJ % 4 == 0 && 16 * HI * 4 * V * nt::kThreads <= sizeof(sm), "stage");
  f32x4* stage = reinterpret_cast<f32x4*>(&sm) + threadIdx.x;
  const int64_t col = j0 + G::col_of();
  const int64_t r8 = (a.rows + 7) / 8 * 8, c8 = (a.cols + 7) / 8 * 8;
  const int wide = (int)min((int64_t)TJ, max((int64_t)0, c8 - col));  // columns stored (zeros among them)
#pragma unroll
  for (int h = 0; h < TI / HI; ++h) {
#pragma unroll
    for (int i = 0; i < HI; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int v = 0; v < V; ++v)
          stage[((i * 4 + r) * V + v) * nt::kThreads] =
              f32x4{acc[h * HI + i][4 * v][r], acc[h * HI + i][4 * v + 1][r], acc[h * HI + i][4 * v + 2][r],
                    acc[h * HI + i][4 * v + 3][r]};
#pragma unroll 1
    for (int q = 0; q < HI; ++q) {
      const int64_t row = i0 + G::row_of(h * HI + q, 0);  // four rows, TJ columns
      if (row >= r8 || wide <= 0) continue;
      float f[4][TJ];
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const f32x4 x = stage[((q * 4 + r) * V + v) * nt::kThreads];
#pragma unroll
          for (int e = 0; e < 4; ++e) f[r][4 * v + e] = a.alpha * x[e];
        }
      if (a.D.hi != nullptr) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (row + r < a.rows) {
            const int64_t at = z * a.D.stride + (row + r) * a.D.ld + col;
            if (wide == TJ) {
              uint16_t d[TJ], e[TJ];
              __builtin_memcpy(d, a.D.hi + at, sizeof d);
              if (PARTS == 2) __builtin_memcpy(e, a.D.lo + at, sizeof e);
#pragma unroll
              for (int j = 0; j < TJ; ++j) f[r][j] += a.beta * (f16_f32(d[j]) + (PARTS == 2 ? f16_f32(e[j]) : 0.0f));
            } else {
#pragma unroll
              for (int j = 0; j < TJ; ++j)
                if (j < wide)
                  f[r][j] += a.beta * (f16_f32(a.D.hi[at + j]) + (PARTS == 2 ? f16_f32(a.D.lo[at + j]) : 0.0f));
            }
          }
      }
      if (a.user != nullptr) {
        const int64_t base = z * a.su;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int j = 0; j < TJ; ++j)
            if (row + r < a.rows && col + j < a.cols) {
              const int64_t at = base + (row + r) * a.si + (col + j) * a.sj;
              if (a.bf16)
                ((bf16_t*)a.user)[at] = f32_to_bf16(f[r][j]);
              else
                ((float*)a.user)[at] = f[r][j];
            }
        continue;
      }
      uint16_t hi[4][TJ], lo[4][TJ];
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
          hi[r][j] = f16_bits(f[r][j]);
          lo[r][j] = PARTS == 2 ? f16_bits(f[r][j] - f16_f32(hi[r][j])) : (uint16_t)0;
        }
      // by rows: TJ consecutive columns of each
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (row + r < a.rows) {
          const int64_t at = z * a.o.stride + (row + r) * a.o.ld + col;
          if (wide == TJ) {
            __builtin_memcpy(a.o.hi + at, hi[r], sizeof hi[r]);
            if (PARTS == 2) __builtin_memcpy(a.o.lo + at, lo[r], sizeof lo[r]);
          } else {
#pragma unroll
            for (int j = 0; j < TJ; ++j)
              if (j < wide) {
                a.o.hi[at + j] = hi[r][j];
                if (PARTS == 2) a.o.lo[at + j] = lo[r][j];
              }
          }
        }
      // by columns: four consecutive rows of each (rows of `t` hold r8 entries)
      if (SYM ? ti != tj : a.t.hi != nullptr) {
        const Parts& t = SYM ? a.o : a.t;
#pragma unroll
        for (int j = 0; j < TJ; ++j)
          if (col + j < a.cols) {
            const int64_t at = z * t.stride + (col + j) * t.ld + row;
            const uint16_t vh[4] = {hi[0][j], hi[1][j], hi[2][j], hi[3][j]};
            put4(t.hi + at, vh);
            if (PARTS == 2) {
              const uint16_t vl[4] = {lo[0][j], lo[1][j], lo[2][j], lo[3][j]};
              put4(t.lo + at, vl);
            }
          }
      }
    }
  }
}

template <int PARTS, bool SYM>
hipError_t step_for(StepArgs a, int64_t batch, hipStream_t s) {
  auto tiles = [&](int64_t b) {
    const int64_t mt = (a.rows + b - 1) / b, ntl = (a.cols + b - 1) / b;
    return SYM ? mt * (mt + 1) / 2 : mt * ntl;
  };
  const bool big = tiles(256) * batch >= 128;
  const int b = big ? 256 : 128;
  a.mt = (int)((a.rows + b - 1) / b);
  a.ntl = (int)((a.cols + b - 1) / b);
  const int64_t wgs = tiles(b);
  if (wgs > 0x7fffffff || batch > 65535) return hipErrorInvalidValue;
  const dim3 grid((uint32_t)wgs, (uint32_t)batch);
  if (big)
    hipLaunchKernelGGL((k_step<PARTS, 8, 8, SYM>), grid, dim3(nt::kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((k_step<PARTS, 4, 4, SYM>), grid, dim3(nt::kThreads), 0, s, a);
  return hipGetLastError();
}

// Largest |b u + c u^2| for u in [0, top].
double quad_bound(double b, double c, double top) {
  double v = fabs(b * top + c * top * top);
  if (c != 0.0) {
    const double u = -b / (2.0 * c);
    if (u > 0.0 && u < top) v = std::max(v, fabs(b * u + c * u * u));
  }
  return v;
}
// Largest |s (a + b s^2 + c s^4)| for s in [0, top].
double poly_bound(double a, double b, double c, double top) {
  auto f = [&](double s) { return fabs(s * (a + b * s * s + c * s * s * s * s)); };
  double v = f(top);
  // stationary where a + 3 b u + 5 c u^2 = 0, u = s^2
  const double qa = 5.0 * c, qb = 3.0 * b, d = qb * qb - 4.0 * qa * a;
  auto at = [&](double u) {
    if (u > 0.0 && u < top * top) v = std::max(v, f(sqrt(u)));
  };
  if (qa == 0.0) {
    if (qb != 0.0) at(-a / qb);
  } else if (d >= 0.0) {
    at((-qb + sqrt(d)) / (2.0 * qa));
    at((-qb - sqrt(d)) / (2.0 * qa));
  }
  return v;
}
// Bound of all iterates' singular values.
double iterates_bound(int steps, double a, double b, double c) {
  double top = 1.0, most = 1.0;
  for (int k = 0; k < steps; ++k) {
    top = poly_bound(a, b, c, top);
    most = std::max(most, top);
    if (!(most < 1e6)) return INFINITY;
  }
  return most;
}
// The power of two that takes numbers up to `bound` to at most 2^15 (half of
// fp16's range; rounding adds less than the other half).
float scale_for(double bound) {
  int e;
  frexp(std::max(bound, 1e-3), &e);  // bound < 2^e
  return ldexpf(1.0f, 15 - e);
}

struct Buffers {
  double* part;
  Parts x[2], t[2], gram, poly;
  size_t bytes;
};
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

Buffers layout(int64_t batch, int64_t m, int64_t n, int parts, char* base) {
  const int64_t r = std::min(m, n), c = std::max(m, n);
  const int64_t ldc = (c + 63) / 64 * 64, ldr = (r + 63) / 64 * 64;
  Buffers b{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* p = base + off;
    off += up256(bytes);
    return p;
  };
  auto operand = [&](int64_t rows, int64_t ld) {
    Parts p{};
    p.ld = ld;
    p.stride = rows * ld;
    p.hi = (uint16_t*)take((size_t)(batch * p.stride) * 2);
    if (parts == 2) p.lo = (uint16_t*)take((size_t)(batch * p.stride) * 2);
    return p;
  };
  b.part = (double*)take((size_t)batch * kNormParts * sizeof(double));
  for (int k = 0; k < 2; ++k) {
    b.x[k] = operand(r, ldc);
    b.t[k] = operand(c, ldr);
  }
  b.gram = operand(r, ldr);
  b.poly = operand(r, ldr);
  b.bytes = off;
  return b;
}

template <int PARTS, class E>
hipError_t run(const OrthoArgs& a, void* workspace, hipStream_t s) {
  const bool tall = a.m > a.n;
  const int64_t r = std::min(a.m, a.n), c = std::max(a.m, a.n);
  Buffers w = layout(a.batch, a.m, a.n, PARTS, (char*)workspace);
  const double most = iterates_bound(a.steps, a.a, a.b, a.c);
  const float sx = scale_for(most), sa = scale_for(most * most), sb = scale_for(quad_bound(a.b, a.c, most * most));
  const int parts = (int)std::min<int64_t>(kNormParts, (a.m * ((a.n + 7) / 8) + 255) / 256);
  hipLaunchKernelGGL(k_square_sums<E>, dim3((uint32_t)parts, (uint32_t)a.batch), dim3(256), 0, s, (const E*)a.g,
                     a.ldg, a.sg, a.m, a.n, w.part);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_start<E, PARTS>),
                     dim3((uint32_t)((a.n + 63) / 64), (uint32_t)((a.m + 63) / 64), (uint32_t)a.batch), dim3(256), 0,
                     s, (const E*)a.g, a.ldg, a.sg, a.m, a.n, w.part, parts, (double)a.eps, sx,
                     tall ? w.t[0] : w.x[0], tall ? w.x[0] : w.t[0]);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const int64_t r8 = (r + 7) / 8 * 8, c8 = (c + 7) / 8 * 8;
  for (int k = 0; k < a.steps; ++k) {
    const int cur = k & 1, nxt = cur ^ 1;
    StepArgs q{};
    q.rows = q.cols = r;
    q.k = c8;
    q.L = q.R = w.x[cur];
    q.o = w.gram;
    q.alpha = sa / (sx * sx);
    if ((e = step_for<PARTS, true>(q, a.batch, s)) != hipSuccess) return e;
    q.k = r8;
    q.L = q.R = q.D = w.gram;
    q.o = w.poly;
    q.alpha = a.c * sb / (sa * sa);
    q.beta = a.b * sb / sa;
    if ((e = step_for<PARTS, true>(q, a.batch, s)) != hipSuccess) return e;
    q.cols = c;
    q.L = w.poly;
    q.R = w.t[cur];
    q.D = w.x[cur];
    q.o = w.x[nxt];
    q.t = w.t[nxt];
    q.alpha = 1.0f / sb;
    q.beta = a.a;
    if (k + 1 == a.steps) {
      q.alpha *= a.scale / sx;
      q.beta *= a.scale / sx;
      q.user = a.out;
      q.si = tall ? 1 : a.ldo;
      q.sj = tall ? a.ldo : 1;
      q.su = a.so;
      q.bf16 = a.bf16;
    }
    if ((e = step_for<PARTS, false>(q, a.batch, s)) != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

bool ortho_bounded(int steps, double a, double b, double c) { return iterates_bound(steps, a, b, c) < 16.0; }

size_t ortho_workspace(int64_t batch, int64_t m, int64_t n, bool bf16) {
  return layout(batch, m, n, bf16 ? 1 : 2, nullptr).bytes;
}

hipError_t launch_ortho(const OrthoArgs& a, void* workspace, hipStream_t s) {
  // 2^20: the operands' rows stay within nt::kMaxRowBytes, the grid within its limits
  if (a.batch <= 0 || a.batch > 65535 || a.m <= 0 || a.n <= 0 || std::max(a.m, a.n) > (1 << 20) || a.steps <= 0 ||
      workspace == nullptr || (uintptr_t)workspace % 256 != 0 || !ortho_bounded(a.steps, a.a, a.b, a.c))
    return hipErrorInvalidValue;
  return a.bf16 ? run<1, bf16_t>(a, workspace, s) : run<2, float>(a, workspace, s);
}

}  // namespace ff
