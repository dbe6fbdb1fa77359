// Orthogonalisation of an update by Newton-Schulz products:
//   X = G / (||G||_F + eps);  X <- a X + (b A + c A A) X with A = X X^T,
// an odd polynomial of X's singular values that takes them towards 1 and
// leaves its singular vectors.  X is r x c with r <= c (a tall G is taken
// transposed), so the two symmetric products are of the smaller side.
//
// The products run on the matrix cores in fp16: the operands are bounded (X's
// singular values by the polynomial's range, known on the host), so a fixed
// power of two per operand puts them where fp16 keeps 11 bits, three more than
// bf16 at the same rate.  For fp32 updates every operand is held as hi + lo (22
// bits) and a product is three, hi hi + hi lo + lo hi, the k axis running over
// them one after the other; lo lo, 2^-22 of the product, is left out.  For bf16
// updates the products take one part each, but the a X that is added keeps both
// of X: what rounding X puts into directions that the update hardly has grows by
// a a step (3.44^5 = 485 over five) through a X alone, for b A + c A A is small
// there, while errors of a product stay within the update's own directions.  A
// matrix of rank 16 was off by 4e-2 with X in one part throughout, by 1.9e-3 so,
// of which 1.7e-3 is the result's own rounding; the most of 84 measured, an eighth
// of 300 x 1000's rows over zeros, by 3.3e-3.  The last step adds X in one part:
// a 2^-12 of it at most, below the result's rounding.  All sums are fp32.
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

constexpr int kNormParts = 1024;  // partial sums of squares per matrix

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
// it is and transposed, each in the parts it has, zeros up to the next multiple
// of eight.
template <class E>
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
    if (o.lo != nullptr) *reinterpret_cast<u32x4*>(o.lo + at) = lo;
  }
}

// One product of a step, C = L R^T with L: rows x k, R: cols x k.
//   out = alpha C + beta D, D (nullable) laid out as C, in parts;
// stored by rows (o) and by columns (t), or as the result (user, E), or, k in
// `splits` parts, as partial sums (sums: splits x batch x rows x c8 fp32).
// Large ones are bound by the matrix cores (the product with X of a 4096 x 11008
// bf16 update: 317 us for the last step, 1.16 PFLOP/s, 688 tiles of 256 x 256 making
// 2.7 rounds; 371 to 394 for the others, X's second part read and written), small
// ones by a kernel's start, first reads and stores (5 to 7 us).
// 3 x 1500 x 1000 fp32, three fp16 products: 26 to 33 us for a symmetric one
// (tiles of 64 x 64: 408), 49 to 56 for the one with X, whose D and
// results in parts and both ways are 54 MB, 11 us at a copy's rate.
struct StepArgs {
  int64_t rows, cols, k;  // k a multiple of 8 (the operands' zeros included)
  Parts L, R, D, o, t;
  float alpha, beta;
  void* user;  // the result: element (i, j) at i si + j sj
  int64_t si, sj, su;
  int bf16;
  int mt, ntl, tiles;  // tile rows and columns, tiles in all
  int splits;
  float* sums;
};

// N consecutive fp16 numbers of a row, as they lie in memory.
template <int N>
struct Halves {
  uint32_t w[N / 2];
  __device__ __forceinline__ float get(int j) const { return f16_f32((uint16_t)(w[j >> 1] >> (16 * (j & 1)))); }
  __device__ __forceinline__ void load(const uint16_t* p, int count) {
    if (count >= N) {
      __builtin_memcpy(w, p, sizeof w);
    } else {
#pragma unroll
      for (int q = 0; q < N / 2; ++q) w[q] = 0;
#pragma unroll
      for (int j = 0; j < N - 1; ++j)
        if (j < count) w[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
    }
  }
  __device__ __forceinline__ void store(uint16_t* p, int count) const {
    if (count >= N) {
      __builtin_memcpy(p, w, sizeof w);
    } else {
#pragma unroll
      for (int j = 0; j < N - 1; ++j)
        if (j < count) p[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
    }
  }
};
// f[0] .. f[N - 1] rounded, and what the rounding left, rounded.
template <int N>
__device__ __forceinline__ void split_parts(const float (&f)[N], Halves<N>& hi, Halves<N>& lo) {
#pragma unroll
  for (int q = 0; q < N / 2; ++q) {
    const uint16_t a = f16_bits(f[2 * q]), b = f16_bits(f[2 * q + 1]);
    hi.w[q] = (uint32_t)a | ((uint32_t)b << 16);
    lo.w[q] = (uint32_t)f16_bits(f[2 * q] - f16_f32(a)) | ((uint32_t)f16_bits(f[2 * q + 1] - f16_f32(b)) << 16);
  }
}

// Results of four rows from `row` on, N columns from `col` on, into o by rows
// and into t (null: not) by columns.  wide: columns that exist, the zeros up to
// the next multiple of eight among them; rows of t hold zeros likewise.  BOTH: o
// may have two parts, with PARTS == 2 t has too.
template <int PARTS, bool BOTH, int N>
__device__ __forceinline__ void store_parts(const float (&f)[4][N], int64_t row, int64_t rows, int64_t col,
                                            int64_t cols, int wide, const Parts& o, const Parts* t, int64_t z) {
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (row + r < rows) {
      Halves<N> hi, lo;
      split_parts<N>(f[r], hi, lo);
      const int64_t at = z * o.stride + (row + r) * o.ld + col;
      hi.store(o.hi + at, wide);
      if (PARTS == 2 || (BOTH && o.lo != nullptr)) lo.store(o.lo + at, wide);
    }
  if (t == nullptr) return;
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (col + j < cols) {
      const float c[4] = {f[0][j], f[1][j], f[2][j], f[3][j]};
      Halves<4> hi, lo;
      split_parts<4>(c, hi, lo);
      const int64_t at = z * t->stride + (col + j) * t->ld + row;
      hi.store(t->hi + at, 4);
      if (PARTS == 2) lo.store(t->lo + at, 4);
    }
}

// k three times over, for operands in two parts: hi lo, lo hi, then hi hi (the
// largest last).
struct Thrice {
  const char *lh, *rh;  // the larger parts at k = 0
  const char* next;     // L's part of the next round
  int bytes;            // of k
  const char *pa, *pb;
  int left;
  // at pair p of 3 `pairs`
  __device__ __forceinline__ Thrice(const char* lh, const char* ll, const char* rh, const char* rl, int bytes,
                                    int p, int pairs)
      : lh(lh), rh(rh), bytes(bytes) {
    const int round = (p >= pairs) + (p >= 2 * pairs), k = (p - round * pairs) * nt::kPair;
    next = round == 0 ? ll : lh;
    pa = (round == 1 ? ll : lh) + k;
    pb = (round == 0 ? rl : rh) + k;
    left = bytes - k;
  }
  __device__ __forceinline__ int operator()(const char*& a, const char*& b) {
    a = pa;
    b = pb;
    const int l = left;
    const bool end = l <= nt::kPair;
    pa = end ? next : pa + nt::kPair;
    pb = end ? rh : pb + nt::kPair;
    left = end ? bytes : l - nt::kPair;
    next = end ? lh : next;
    return l;
  }
};

template <int PARTS, int TI, int TJ, int SLOTS, bool SYM>
__global__ __launch_bounds__(nt::kThreads, ((TI + TJ) * SLOTS <= 20 ? 2 : 1)) void k_step(StepArgs a) {
  typedef nt::Tile<nt::F16, TI, TJ, SLOTS> G;
  __shared__ typename G::Ring sm;
  const uint32_t w = xcd_remap(blockIdx.x, gridDim.x);
  const uint32_t part = w / a.tiles, tile = w - part * a.tiles;
  uint32_t ti, tj;
  if (SYM) {
    grouped_tile(tile, a.mt, ti, tj);
  } else {
    const uint32_t strip = tile / (8 * a.ntl), u = tile - strip * 8 * a.ntl, r = min(8u, a.mt - strip * 8);
    ti = strip * 8 + u % r;
    tj = u / r;
  }
  const int64_t i0 = (int64_t)ti * G::BM, j0 = (int64_t)tj * G::BN, z = blockIdx.y;
  const nt::Rows A{nullptr, (int)min((int64_t)G::BM, a.rows - i0), (uint32_t)(a.L.ld * 2)};
  const nt::Rows B{nullptr, (int)min((int64_t)G::BN, a.cols - j0), (uint32_t)(a.R.ld * 2)};
  const int64_t la = z * a.L.stride + i0 * a.L.ld, rb = z * a.R.stride + j0 * a.R.ld;
  const int kbytes = (int)a.k * 2, pairs = (kbytes + nt::kPair - 1) / nt::kPair;
  const int total = PARTS == 2 ? 3 * pairs : pairs;
  const int64_t col = j0 + G::col_of(), first = i0 + G::row_of(0, 0);
  const int64_t r8 = (a.rows + 7) / 8 * 8, c8 = (a.cols + 7) / 8 * 8;
  const int wide = (int)min((int64_t)TJ, max((int64_t)0, c8 - col));
  Halves<TJ> dh[4], dl[4];
  // (of the products of one part, the one with X adds both of X)
  constexpr bool BOTH = PARTS == 2 || !SYM;
  const bool add = a.D.hi != nullptr && a.sums == nullptr && wide > 0;
  const bool low = PARTS == 2 || (BOTH && a.D.lo != nullptr);
  auto fetch = [&](int i) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t at = z * a.D.stride + min(first + i * 16 + r, a.rows - 1) * a.D.ld + col;
      dh[r].load(a.D.hi + at, wide);
      if (BOTH && low) dl[r].load(a.D.lo + at, wide);
    }
  };
  if (add) fetch(0);  // (lands during the loop)
  typename G::Acc acc;
  G::zero(acc);
  const int p0 = (int)((int64_t)total * part / a.splits), p1 = (int)((int64_t)total * (part + 1) / a.splits);
  if (PARTS == 1) {
    nt::Straight walk{(const char*)(a.L.hi + la) + p0 * nt::kPair, (const char*)(a.R.hi + rb) + p0 * nt::kPair,
                      kbytes - p0 * nt::kPair};
    G::loop(sm, A, B, p1 - p0, walk, acc);
  } else {
    Thrice walk{(const char*)(a.L.hi + la), (const char*)(a.L.lo + la), (const char*)(a.R.hi + rb),
                (const char*)(a.R.lo + rb), kbytes, p0, pairs};
    G::loop(sm, A, B, p1 - p0, walk, acc);
  }
  // through LDS and four rows at a time, as in the linear layers
  constexpr int HI = TI < 4 ? TI : TI % 4 == 0 ? 4 : 3, PC = TJ % 4 == 0 ? 4 : 2, V = TJ / PC;
  typedef __attribute__((ext_vector_type(PC))) float Slot;
  static_assert(TI % HI == 0 && TJ % 2 == 0 && sizeof(Slot) * HI * 4 * V * nt::kThreads <= sizeof(sm), "stage");
  Slot* stage = reinterpret_cast<Slot*>(&sm) + threadIdx.x;
#pragma unroll
  for (int h = 0; h < TI / HI; ++h) {
#pragma unroll
    for (int i = 0; i < HI; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          Slot s;
#pragma unroll
          for (int e = 0; e < PC; ++e) s[e] = acc[h * HI + i][PC * v + e][r];
          stage[((i * 4 + r) * V + v) * nt::kThreads] = s;
        }
#pragma unroll 1
    for (int q = 0; q < HI; ++q) {
      const int i = h * HI + q;
      const int64_t row = first + i * 16;  // four rows, TJ columns
      float f[4][TJ];
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const Slot s = stage[((q * 4 + r) * V + v) * nt::kThreads];
#pragma unroll
          for (int e = 0; e < PC; ++e) f[r][PC * v + e] = s[e];
        }
      if (a.sums != nullptr) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (row + r < a.rows) {
            float* o = a.sums + (((int64_t)part * gridDim.y + z) * a.rows + row + r) * c8 + col;
            if (wide == TJ) {
              __builtin_memcpy(o, f[r], sizeof f[r]);
            } else {
#pragma unroll
              for (int j = 0; j < TJ - 1; ++j)
                if (j < wide) o[j] = f[r][j];
            }
          }
        continue;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < TJ; ++j) f[r][j] *= a.alpha;
      if (add) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float b = row + r < a.rows ? a.beta : 0.0f;  // (rows beyond: zeros, not the last row's)
#pragma unroll
          for (int j = 0; j < TJ; ++j) f[r][j] += b * (dh[r].get(j) + (PARTS == 2 ? dl[r].get(j) : 0.0f));
          if (PARTS == 1 && BOTH && low) {
#pragma unroll
            for (int j = 0; j < TJ; ++j) f[r][j] += b * dl[r].get(j);
          }
        }
        if (i + 1 < TI) fetch(i + 1);
      }
      if (row >= r8 || wide <= 0) continue;
      if (a.user == nullptr) {
        const Parts& t = SYM ? a.o : a.t;
        store_parts<PARTS, BOTH, TJ>(f, row, a.rows, col, a.cols, wide, a.o, !SYM || ti != tj ? &t : nullptr, z);
        continue;
      }
      const int64_t base = z * a.su;
      const bool inside = row + 4 <= a.rows && col + TJ <= a.cols;
      if (inside && a.sj == 1) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if (a.bf16) {
            uint32_t o[TJ / 2];
#pragma unroll
            for (int j = 0; j < TJ / 2; ++j)
              o[j] = (uint32_t)f32_to_bf16(f[r][2 * j]) | ((uint32_t)f32_to_bf16(f[r][2 * j + 1]) << 16);
            __builtin_memcpy((bf16_t*)a.user + base + (row + r) * a.si + col, o, sizeof o);
          } else {
            __builtin_memcpy((float*)a.user + base + (row + r) * a.si + col, f[r], sizeof f[r]);
          }
        }
      } else if (inside && a.si == 1) {
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
          const int64_t at = base + row + (col + j) * a.sj;
          if (a.bf16) {
            const uint32_t o[2] = {(uint32_t)f32_to_bf16(f[0][j]) | ((uint32_t)f32_to_bf16(f[1][j]) << 16),
                                   (uint32_t)f32_to_bf16(f[2][j]) | ((uint32_t)f32_to_bf16(f[3][j]) << 16)};
            __builtin_memcpy((bf16_t*)a.user + at, o, sizeof o);
          } else {
            const float o[4] = {f[0][j], f[1][j], f[2][j], f[3][j]};
            __builtin_memcpy((float*)a.user + at, o, sizeof o);
          }
        }
      } else {
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
      }
    }
  }
}

// The symmetric product's partial sums (tiles of `edge` on and above the
// diagonal) added in their order: four columns of a row a thread, those below
// the diagonal's tiles read across it.
template <int PARTS>
__global__ __launch_bounds__(256) void k_step_join(StepArgs a, int edge) {
  const int64_t c8 = (a.cols + 7) / 8 * 8, q4 = c8 / 4, z = blockIdx.y;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, row = id / q4, col = id % q4 * 4;
  if (row >= a.rows) return;
  const bool upper = row / edge <= col / edge;
  const int64_t step = (int64_t)gridDim.y * a.rows * c8;
  const float* p = a.sums + z * a.rows * c8;
  float f[4] = {};
#pragma unroll 4
  for (int s = 0; s < a.splits; ++s) {
    float v[4] = {};
    if (upper) {
      __builtin_memcpy(v, p + s * step + row * c8 + col, 16);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (col + j < a.rows) v[j] = p[s * step + (col + j) * c8 + row];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] += v[j];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) f[j] *= a.alpha;
  Halves<4> hi, lo;
  split_parts<4>(f, hi, lo);
  const int64_t at = z * a.o.stride + row * a.o.ld + col;
  hi.store(a.o.hi + at, 4);
  if (PARTS == 2) lo.store(a.o.lo + at, 4);
}

// The fastest form of a product by a model of the forms' times (us), as for the
// linear layers: per pair of k `pair` with a compute unit to itself, `loaded`
// with all of them busy, `ends` for a tile's start and epilogue.  (Predicts too little
// where tiles store both ways: symmetric 4096 with k = 11008 154 us for 192 measured.)
struct StepForm {
  int ti, tj, slots, wgs;
  double pair, loaded, ends;
};
struct StepPlan {
  int form, splits;
};
constexpr StepForm kSymForms[] = {{8, 8, 2, 1, 1.36, 1.36, 12.0}, {6, 6, 2, 1, 0.85, 0.85, 8.0},
                                  {4, 4, 2, 2, 0.53, 0.85, 6.5},  {4, 4, 4, 1, 0.40, 0.53, 5.0},
                                  {2, 2, 5, 2, 0.17, 0.30, 2.0}};
constexpr StepForm kAnyForms[] = {{8, 8, 2, 1, 1.36, 1.36, 12.0}, {6, 8, 2, 1, 1.09, 1.09, 10.0},
                                  {4, 8, 3, 1, 0.79, 0.79, 8.0},  {4, 6, 3, 1, 0.61, 0.61, 7.0},
                                  {4, 4, 2, 2, 0.53, 0.85, 6.5},  {4, 4, 4, 1, 0.40, 0.55, 5.0},
                                  {2, 4, 3, 2, 0.25, 0.50, 3.0}};

StepPlan step_plan(bool sym, bool may_split, int64_t rows, int64_t cols, int64_t k, int64_t batch, int parts) {
  const int64_t pairs = (k * 2 + nt::kPair - 1) / nt::kPair * (parts == 2 ? 3 : 1);
  StepPlan best{0, 1};
  double least = 1e300;
  const int forms = sym ? 5 : 7;
  for (int q = 0; q < forms; ++q) {
    const StepForm& f = sym ? kSymForms[q] : kAnyForms[q];
    const int64_t mt = (rows + 32 * f.ti - 1) / (32 * f.ti), ntl = (cols + 32 * f.tj - 1) / (32 * f.tj);
    const int64_t tiles = (sym ? mt * (mt + 1) / 2 : mt * ntl) * batch;
    for (int s : {1, 2, 4, 8, 16}) {
      if (s > 1 && (!may_split || s * 4 > pairs || tiles * s > 512)) break;
      const int64_t wgs = tiles * s, rounds = (wgs + 256 * f.wgs - 1) / (256 * f.wgs);
      double us = (double)rounds * (f.ends + (double)((pairs + s - 1) / s) * (wgs > 256 ? f.loaded : f.pair));
      if (s > 1) us += 6.0 + 8.0 * (double)s * (double)(batch * rows * rows) / 4e6;
      if (us < least) {
        least = us;
        best = {q, s};
      }
    }
  }
  return best;
}

template <int PARTS, int TI, int TJ, int SLOTS, bool SYM>
hipError_t step_tiles(StepArgs a, int64_t batch, hipStream_t s) {
  constexpr int BM = 32 * TI, BN = 32 * TJ;
  a.mt = (int)((a.rows + BM - 1) / BM);
  a.ntl = (int)((a.cols + BN - 1) / BN);
  const int64_t tiles = SYM ? (int64_t)a.mt * (a.mt + 1) / 2 : (int64_t)a.mt * a.ntl;
  if (tiles * a.splits > 0x7fffffff || batch > 65535) return hipErrorInvalidValue;
  a.tiles = (int)tiles;
  hipLaunchKernelGGL((k_step<PARTS, TI, TJ, SLOTS, SYM>), dim3((uint32_t)(tiles * a.splits), (uint32_t)batch),
                     dim3(nt::kThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t threads = a.rows * ((a.cols + 7) / 8 * 2);
  hipLaunchKernelGGL(k_step_join<PARTS>, dim3((uint32_t)((threads + 255) / 256), (uint32_t)batch), dim3(256), 0, s, a,
                     BM);
  return hipGetLastError();
}

template <int PARTS>
hipError_t sym_step(StepArgs a, int form, int splits, float* sums, int64_t batch, hipStream_t s) {
  a.splits = splits;
  a.sums = splits > 1 ? sums : nullptr;
  switch (form) {
    case 0: return step_tiles<PARTS, 8, 8, 2, true>(a, batch, s);
    case 1: return step_tiles<PARTS, 6, 6, 2, true>(a, batch, s);
    case 2: return step_tiles<PARTS, 4, 4, 2, true>(a, batch, s);
    case 3: return step_tiles<PARTS, 4, 4, 4, true>(a, batch, s);
    default: return step_tiles<PARTS, 2, 2, 5, true>(a, batch, s);
  }
}
template <int PARTS>
hipError_t any_step(StepArgs a, int form, int64_t batch, hipStream_t s) {
  a.splits = 1;
  switch (form) {
    case 0: return step_tiles<PARTS, 8, 8, 2, false>(a, batch, s);
    case 1: return step_tiles<PARTS, 6, 8, 2, false>(a, batch, s);
    case 2: return step_tiles<PARTS, 4, 8, 3, false>(a, batch, s);
    case 3: return step_tiles<PARTS, 4, 6, 3, false>(a, batch, s);
    case 4: return step_tiles<PARTS, 4, 4, 2, false>(a, batch, s);
    case 5: return step_tiles<PARTS, 4, 4, 4, false>(a, batch, s);
    default: return step_tiles<PARTS, 2, 4, 3, false>(a, batch, s);
  }
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
  float* sums;  // partial sums of the first product
  Parts x[2], t[2], gram, poly;  // x: always in two parts
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
  auto operand = [&](int64_t rows, int64_t ld, int parts) {
    Parts p{};
    p.ld = ld;
    p.stride = rows * ld;
    p.hi = (uint16_t*)take((size_t)(batch * p.stride) * 2);
    if (parts == 2) p.lo = (uint16_t*)take((size_t)(batch * p.stride) * 2);
    return p;
  };
  b.part = (double*)take((size_t)batch * kNormParts * sizeof(double));
  for (int k = 0; k < 2; ++k) {
    b.x[k] = operand(r, ldc, 2);
    b.t[k] = operand(c, ldr, parts);
  }
  const int splits = ortho_plan(batch, m, n, parts == 1).gram_splits;
  if (splits > 1) b.sums = (float*)take((size_t)splits * (size_t)(batch * r * ((r + 7) / 8 * 8)) * sizeof(float));
  b.gram = operand(r, ldr, parts);
  b.poly = operand(r, ldr, parts);
  b.bytes = off;
  return b;
}

// ------------------------------------------------------------ small matrices
// All steps of one matrix in one workgroup of 16 waves, everything in LDS: X by
// rows and by columns and one r x r matrix (A, then b A + c A A in its place),
// each in PARTS fp16 parts with rows of whole 64-byte steps of k plus 16 bytes
// (16 consecutive rows at one k then start in different banks).  A wave takes
// whole 16 x 16 tiles; what it computes replaces an operand of the others, so
// it stays in registers until all of them are done (LIMIT tiles a wave).  The
// matrices are symmetric: a lane's four consecutive rows of one column are stored
// as four consecutive columns of one row.  Bound by LDS reads and their latency:
// 64 x 128 fp32 in 30 us, 4.5 a step and 8 around them, where the launches of the
// larger sizes' way are 17 of 5 to 7 us.
constexpr int kSmallThreads = 1024;
constexpr int small_tiles(int parts) { return parts == 2 ? 4 : 8; }  // a wave, what LDS holds
constexpr size_t kSmallLds = 160 * 1024 - 256;

struct SmallLayout {
  int rp, cp;        // rows of X and X^T: multiples of 16
  int ldx, ldr;      // elements
  size_t x, t, a, bytes;  // parts of X, X^T and A: offsets of the first, bytes of one
};
__host__ __device__ inline SmallLayout small_layout(int r, int c, int parts) {
  SmallLayout s{};
  s.rp = (r + 15) / 16 * 16;
  s.cp = (c + 15) / 16 * 16;
  s.ldx = (c + 31) / 32 * 32 + 8;
  s.ldr = (r + 31) / 32 * 32 + 8;
  s.x = (size_t)s.rp * s.ldx * 2;
  s.t = (size_t)s.cp * s.ldr * 2;
  s.a = (size_t)s.rp * s.ldr * 2;
  s.bytes = (s.x + s.t + s.a) * (size_t)parts;
  return s;
}
bool small_fits(int64_t m, int64_t n, int parts) {
  const int64_t r = std::min(m, n), c = std::max(m, n);
  if (c > 4096) return false;
  const SmallLayout s = small_layout((int)r, (int)c, parts);
  return s.bytes <= kSmallLds && (s.rp / 16) * (s.cp / 16) <= small_tiles(parts) * (kSmallThreads / 64);
}

// Parts with which a matrix is taken here, 0: not at all.  Two where they fit,
// for bf16 too: few directions average few roundings (128 x 128 is off by up to
// 3.0e-3 with one part, 96 x 80 by its own rounding, 1.7e-3, with two).  With one,
// what X's rounding leaves of a wave's own tiles stays in its registers.
int small_parts(int64_t m, int64_t n, bool bf16) { return small_fits(m, n, 2) ? 2 : bf16 && small_fits(m, n, 1) ? 1 : 0; }

struct SmallArgs {
  int r, c, steps, tall, bf16;
  const void* g;
  int64_t ldg, sg;
  void* out;
  int64_t ldo, so;
  float a, b, c5, scale, sx, sa, sb;  // coefficients, the result's scale, the operands' scales
  double eps;
};

template <class E, int PARTS>
__global__ __launch_bounds__(kSmallThreads) void k_small(SmallArgs a) {
  extern __shared__ char lds[];
  __shared__ double share[kSmallThreads / 64];
  const SmallLayout S = small_layout(a.r, a.c, PARTS);
  char* const X = lds;
  char* const T = X + S.x * PARTS;
  char* const A = T + S.t * PARTS;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  constexpr int W = kSmallThreads / 64, LIMIT = small_tiles(PARTS);
  const E* g = (const E*)a.g + blockIdx.x * a.sg;
  const int m = a.tall ? a.c : a.r, n = a.tall ? a.r : a.c;
  for (size_t o = (size_t)tid * 16; o < S.bytes; o += kSmallThreads * 16) *reinterpret_cast<u32x4*>(lds + o) = u32x4{0, 0, 0, 0};
  // f(row, column, value) of this thread's elements of G, eight loads at a time
  auto elements = [&](auto f) {
    int i[8], j[8];
    i[0] = tid / n;
    j[0] = tid - i[0] * n;
    const int di = kSmallThreads / n, dj = kSmallThreads - di * n;
    for (int id = tid; id < m * n; id += 8 * kSmallThreads) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (k > 0) {
          i[k] = i[k - 1] + di;
          j[k] = j[k - 1] + dj;
          if (j[k] >= n) {
            j[k] -= n;
            ++i[k];
          }
        }
        v[k] = i[k] < m ? Elem<E>::to_f32(g[(int64_t)i[k] * a.ldg + j[k]]) : 0.0f;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (i[k] < m) f(i[k], j[k], v[k]);
      i[0] = i[7] + di;
      j[0] = j[7] + dj;
      if (j[0] >= n) {
        j[0] -= n;
        ++i[0];
      }
    }
  };
  double ss = 0.0;
  elements([&](int, int, float v) { ss += (double)v * (double)v; });
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) ss += __shfl_xor(ss, d);
  if (lane == 0) share[wave] = ss;
  __syncthreads();
  ss = 0.0;
  for (int k = 0; k < W; ++k) ss += share[k];
  const double inv = 1.0 / (sqrt(ss) + a.eps);
  // part q of element (i, j) of a matrix whose parts are `size` bytes apart
  auto at = [](char* M, size_t size, int ld, int q, int i, int j) {
    return reinterpret_cast<uint16_t*>(M + q * size) + i * ld + j;
  };
  elements([&](int gi, int gj, float x) {
    const int i = a.tall ? gj : gi, j = a.tall ? gi : gj;
    const float v = (float)((double)x * inv) * a.sx;
    const uint16_t hi = f16_bits(v), lo = f16_bits(v - f16_f32(hi));
    *at(X, S.x, S.ldx, 0, i, j) = *at(T, S.t, S.ldr, 0, j, i) = hi;
    if (PARTS == 2) *at(X, S.x, S.ldx, 1, i, j) = *at(T, S.t, S.ldr, 1, j, i) = lo;
  });
  __syncthreads();
  // Everything below addresses bytes: a lane's place in a tile plus the tile's
  // (uniform) place in its matrix.
  const int rt = S.rp / 16, ct = S.cp / 16, kr = S.ldr - 8, kc = S.ldx - 8;
  const int lr = 4 * (lane >> 4), lc = lane & 15;  // a lane's first row and its column in a result
  const uint32_t frag_x = (uint32_t)(lc * S.ldx + 2 * lr) * 2, frag_r = (uint32_t)(lc * S.ldr + 2 * lr) * 2;
  const uint32_t four_r = (uint32_t)(lc * S.ldr + lr) * 2, one_x = (uint32_t)(lr * S.ldx + lc) * 2;
  // a 16 x 16 tile of P Q^T from the operands' fragments at p and q, k elements
  auto product = [&](const char* p, size_t ps, const char* q, size_t qs, int k) {
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f}, low = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int kk = 0; kk < k; kk += 32, p += 64, q += 64) {
      const u32x4 ph = *reinterpret_cast<const u32x4*>(p), qh = *reinterpret_cast<const u32x4*>(q);
      if (PARTS == 2) {
        const u32x4 pl = *reinterpret_cast<const u32x4*>(p + ps), ql = *reinterpret_cast<const u32x4*>(q + qs);
        low = nt::F16::mfma(ph, ql, low);
        low = nt::F16::mfma(pl, qh, low);
      }
      acc = nt::F16::mfma(ph, qh, acc);
    }
    return acc + low;
  };
  // With one part: what X's rounding left of this wave's tiles of X
  Halves<4> low[PARTS == 1 ? LIMIT : 1];
  auto put4 = [&](char* p, size_t size, const float (&f)[4]) {
    Halves<4> hi, lo;
    split_parts<4>(f, hi, lo);
    __builtin_memcpy(p, hi.w, 8);
    if (PARTS == 2) __builtin_memcpy(p + size, lo.w, 8);
  };
  auto get4 = [&](const char* p, size_t size, float (&f)[4]) {
    Halves<4> hi, lo;
    __builtin_memcpy(hi.w, p, 8);
    if (PARTS == 2) __builtin_memcpy(lo.w, p + size, 8);
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = hi.get(e) + (PARTS == 2 ? lo.get(e) : 0.0f);
  };
  // (opaque, or every tile's addresses are computed ahead and held)
  auto tile_of = [&](int u) {
    int q = wave + u * W;
    asm volatile("" : "+s"(q));
    return q;
  };
  // q / n and q % n for q < 256 by n's reciprocal in 16 bits
  const uint32_t inv_rt = (65535u + (uint32_t)rt) / (uint32_t)rt, inv_ct = (65535u + (uint32_t)ct) / (uint32_t)ct;
  auto place = [](int q, int n, uint32_t inv, int& i, int& j) {
    i = (int)(((uint32_t)q * inv) >> 16);
    j = q - i * n;
  };
  const int row_x = 16 * S.ldx * 2, row_r = 16 * S.ldr * 2;  // bytes of sixteen rows
  if (PARTS == 1) {
#pragma unroll
    for (int u = 0; u < LIMIT; ++u) {
      const int q = tile_of(u);
      if (q < rt * ct) {
        int i, j;
        place(q, ct, inv_ct, i, j);
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int gi = i * 16 + lr + e, gj = j * 16 + lc;
          const int row = a.tall ? gj : gi, col = a.tall ? gi : gj;
          v[e] = gi < a.r && gj < a.c ? (float)((double)Elem<E>::to_f32(g[(int64_t)row * a.ldg + col]) * inv) * a.sx : 0.0f;
        }
        Halves<4> hi;
        split_parts<4>(v, hi, low[u]);
      }
    }
  }
  const float gram = a.sa / (a.sx * a.sx), square = a.c5 * a.sb / (a.sa * a.sa), keep_a = a.b * a.sb / a.sa,
              back = 1.0f / a.sb;
  for (int step = 0; step < a.steps; ++step) {
    for (int q = wave; q < rt * rt; q += W) {
      int i, j;
      place(q, rt, inv_rt, i, j);
      const f32x4 s = product(X + i * row_x + frag_x, S.x, X + j * row_x + frag_x, S.x, kc);
      const float f[4] = {gram * s[0], gram * s[1], gram * s[2], gram * s[3]};
      put4(A + j * row_r + i * 32 + four_r, S.a, f);
    }
    __syncthreads();
    float keep[LIMIT][4];
#pragma unroll
    for (int u = 0; u < LIMIT; ++u) {
      const int q = tile_of(u);
      if (q < rt * rt) {
        int i, j;
        place(q, rt, inv_rt, i, j);
        const f32x4 s = product(A + i * row_r + frag_r, S.a, A + j * row_r + frag_r, S.a, kr);
        float d[4];
        get4(A + j * row_r + i * 32 + four_r, S.a, d);
#pragma unroll
        for (int e = 0; e < 4; ++e) keep[u][e] = square * s[e] + keep_a * d[e];
      }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < LIMIT; ++u) {
      const int q = tile_of(u);
      if (q < rt * rt) {
        int i, j;
        place(q, rt, inv_rt, i, j);
        put4(A + j * row_r + i * 32 + four_r, S.a, keep[u]);
      }
    }
    __syncthreads();
    const bool last = step + 1 == a.steps;
#pragma unroll
    for (int u = 0; u < LIMIT; ++u) {
      const int q = tile_of(u);
      if (q < rt * ct) {
        int i, j;
        place(q, ct, inv_ct, i, j);
        const f32x4 s = product(A + i * row_r + frag_r, S.a, T + j * row_r + frag_r, S.t, kr);
        float d[4];
        get4(T + j * row_r + i * 32 + four_r, S.t, d);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (PARTS == 1 && !last) d[e] += low[u].get(e);
          keep[u][e] = back * s[e] + a.a * d[e];
        }
        if (last) {
          const int gi = i * 16 + lr, gj = j * 16 + lc;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (gi + e < a.r && gj < a.c) {
              const int64_t o =
                  blockIdx.x * a.so + (a.tall ? (int64_t)gj * a.ldo + gi + e : (int64_t)(gi + e) * a.ldo + gj);
              ((E*)a.out)[o] = Elem<E>::from_f32(keep[u][e] * (a.scale / a.sx));
            }
        }
      }
    }
    if (last) break;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < LIMIT; ++u) {
      const int q = tile_of(u);
      if (q < rt * ct) {
        int i, j;
        place(q, ct, inv_ct, i, j);
        Halves<4> hi, lo;
        split_parts<4>(keep[u], hi, lo);
        if (PARTS == 1) low[u] = lo;
        char* t = T + j * row_r + i * 32 + four_r;
        char* x = X + i * row_x + j * 32 + one_x;
        __builtin_memcpy(t, hi.w, 8);
        if (PARTS == 2) __builtin_memcpy(t + S.t, lo.w, 8);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          *reinterpret_cast<uint16_t*>(x + e * S.ldx * 2) = (uint16_t)(hi.w[e >> 1] >> (16 * (e & 1)));
          if (PARTS == 2)
            *reinterpret_cast<uint16_t*>(x + S.x + e * S.ldx * 2) = (uint16_t)(lo.w[e >> 1] >> (16 * (e & 1)));
        }
      }
    }
    __syncthreads();
  }
}

template <int PARTS, class E>
hipError_t run_small(const OrthoArgs& a, float sx, float sa, float sb, hipStream_t s) {
  SmallArgs q{};
  q.tall = a.m > a.n;
  q.r = (int)std::min(a.m, a.n);
  q.c = (int)std::max(a.m, a.n);
  q.steps = a.steps;
  q.g = a.g;
  q.ldg = a.ldg;
  q.sg = a.sg;
  q.out = a.out;
  q.ldo = a.ldo;
  q.so = a.so;
  q.a = a.a;
  q.b = a.b;
  q.c5 = a.c;
  q.scale = a.scale;
  q.sx = sx;
  q.sa = sa;
  q.sb = sb;
  q.eps = a.eps;
  hipLaunchKernelGGL((k_small<E, PARTS>), dim3((uint32_t)a.batch), dim3(kSmallThreads),
                     (uint32_t)small_layout(q.r, q.c, PARTS).bytes, s, q);
  return hipGetLastError();
}

template <int PARTS, class E>
hipError_t run(const OrthoArgs& a, void* workspace, hipStream_t s) {
  const double most = iterates_bound(a.steps, a.a, a.b, a.c);
  const float sx = scale_for(most), sa = scale_for(most * most), sb = scale_for(quad_bound(a.b, a.c, most * most));
  const OrthoPlan plan = ortho_plan(a.batch, a.m, a.n, PARTS == 1);
  if (plan.small == 2) return run_small<2, E>(a, sx, sa, sb, s);
  if constexpr (PARTS == 1)
    if (plan.small == 1) return run_small<1, E>(a, sx, sa, sb, s);
  const bool tall = a.m > a.n;
  const int64_t r = std::min(a.m, a.n), c = std::max(a.m, a.n);
  Buffers w = layout(a.batch, a.m, a.n, PARTS, (char*)workspace);
  // X by rows, as step k takes it: of bf16 updates the last one adds it in one part
  auto x_of = [&](int k) {
    Parts x = w.x[k & 1];
    if (PARTS == 1 && k + 1 == a.steps) x.lo = nullptr;
    return x;
  };
  const int parts = (int)std::min<int64_t>(kNormParts, (a.m * ((a.n + 7) / 8) + 255) / 256);
  hipLaunchKernelGGL(k_square_sums<E>, dim3((uint32_t)parts, (uint32_t)a.batch), dim3(256), 0, s, (const E*)a.g,
                     a.ldg, a.sg, a.m, a.n, w.part);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_start<E>,
                     dim3((uint32_t)((a.n + 63) / 64), (uint32_t)((a.m + 63) / 64), (uint32_t)a.batch), dim3(256), 0,
                     s, (const E*)a.g, a.ldg, a.sg, a.m, a.n, w.part, parts, a.eps, sx,
                     tall ? w.t[0] : x_of(0), tall ? x_of(0) : w.t[0]);
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
    if ((e = sym_step<PARTS>(q, plan.gram, plan.gram_splits, w.sums, a.batch, s)) != hipSuccess) return e;
    q.k = r8;
    q.L = q.R = q.D = w.gram;
    q.o = w.poly;
    q.alpha = a.c * sb / (sa * sa);
    q.beta = a.b * sb / sa;
    if ((e = sym_step<PARTS>(q, plan.square, 1, nullptr, a.batch, s)) != hipSuccess) return e;
    q.cols = c;
    q.L = w.poly;
    q.R = w.t[cur];
    q.D = x_of(k);
    q.o = x_of(k + 1);
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
    if ((e = any_step<PARTS>(q, plan.apply, a.batch, s)) != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

bool ortho_bounded(int steps, double a, double b, double c) { return iterates_bound(steps, a, b, c) < 16.0; }

OrthoPlan ortho_plan(int64_t batch, int64_t m, int64_t n, bool bf16) {
  const int small = small_parts(m, n, bf16), parts = bf16 ? 1 : 2;
  if (small != 0) return {small, 0, 1, 0, 0};
  const int64_t r = std::min(m, n), c = std::max(m, n), r8 = (r + 7) / 8 * 8, c8 = (c + 7) / 8 * 8;
  const StepPlan gram = step_plan(true, true, r, r, c8, batch, parts);
  return {0, gram.form, gram.splits, step_plan(true, false, r, r, r8, batch, parts).form,
          step_plan(false, false, r, c, r8, batch, parts).form};
}

size_t ortho_workspace(int64_t batch, int64_t m, int64_t n, bool bf16) {
  if (ortho_plan(batch, m, n, bf16).small != 0) return 0;
  return layout(batch, m, n, bf16 ? 1 : 2, nullptr).bytes;
}

hipError_t launch_ortho(const OrthoArgs& a, void* workspace, hipStream_t s) {
  // 2^20: the operands' rows stay within nt::kMaxRowBytes, the grid within its limits
  if (a.batch <= 0 || a.batch > 65535 || a.m <= 0 || a.n <= 0 || std::max(a.m, a.n) > (1 << 20) || a.steps <= 0 ||
      (workspace == nullptr && ortho_plan(a.batch, a.m, a.n, a.bf16).small == 0) || (uintptr_t)workspace % 256 != 0 || !ortho_bounded(a.steps, a.a, a.b, a.c))
    return hipErrorInvalidValue;
  return a.bf16 ? run<1, bf16_t>(a, workspace, s) : run<2, float>(a, workspace, s);
}

}  // namespace ff
