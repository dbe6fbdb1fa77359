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
#include "ff_q8.hpp"
#include "ff_tile_nt.hpp"
#include "ff_vec.hpp"

namespace ff {
namespace {

// sigmoid(x) = 1 / (1 + 2^(-x log2 e)) by the exponential and reciprocal
// instructions (one unit in the last place each; 0 below x = -87, 1 far out).  The
// argument's roundings, up to 3 2^-24 |x|, are relative errors of the exponential:
// 2^-19 of an activation at x = -10, 2^-16 where it ends, 1e-36; bf16's own is 2^-9.
constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float sigmoid_of(float minus_x_log2e) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(minus_x_log2e));
}

// gelu: z sigmoid(2 c (z + 0.044715 z^3)), c = sqrt(2 / pi) (the tanh form).
constexpr float kGelu = 1.5957691216057308f, kCube = 0.044715f;

__device__ __forceinline__ float gelu_gate(float z) {
  return sigmoid_of(z * (-kGelu * kLog2e - kGelu * kLog2e * kCube * (z * z)));
}
__device__ __forceinline__ float silu_gate(float z) { return sigmoid_of(-kLog2e * z); }

template <int ACT>
__device__ __forceinline__ float act_as(float z) {
  if (ACT == kActRelu) return z < 0.0f ? 0.0f : z;
  if (ACT == kActSilu) return z * silu_gate(z);
  if (ACT == kActGelu) return z * gelu_gate(z);
  return z;
}
__device__ __forceinline__ float act_of(float z, int act) {
  return act == kActRelu   ? act_as<kActRelu>(z)
         : act == kActSilu ? act_as<kActSilu>(z)
         : act == kActGelu ? act_as<kActGelu>(z)
                           : z;
}
__device__ __forceinline__ float act_slope(float z, int act) {
  if (act == kActRelu) return z > 0.0f ? 1.0f : 0.0f;
  if (act == kActSilu) {
    const float p = silu_gate(z);
    return p * (1.0f + z * (1.0f - p));
  }
  if (act == kActGelu) {
    const float p = gelu_gate(z);
    const float t = z * p * (1.0f - p);  // zero for large |z|, where z^2 may be infinite
    return t == 0.0f ? p : p + t * kGelu * (1.0f + 3.0f * kCube * z * z);
  }
  return 1.0f;
}

// W consecutive outputs of row t from column i on (W = 1 or 4), `count` of
// them inside the matrix.
template <int W>
__device__ __forceinline__ void finish(const LinearArgs& a, int64_t t, int64_t i, const float* acc, int count) {
  if (count <= 0) return;
  float z[W];
  const float st = a.x_scale != nullptr ? a.x_scale[t] : 1.0f;
  bf16_t r[W], b[W];
  if (count >= W) {
    if (a.residual != nullptr) __builtin_memcpy(r, a.residual + t * a.ldr + i, sizeof r);
    if (a.bias != nullptr) __builtin_memcpy(b, a.bias + i, sizeof b);
  } else {
#pragma unroll
    for (int k = 0; k < W; ++k) {
      r[k] = b[k] = 0;
      if (k < count) {
        if (a.residual != nullptr) r[k] = a.residual[t * a.ldr + i + k];
        if (a.bias != nullptr) b[k] = a.bias[i + k];
      }
    }
  }
#pragma unroll
  for (int k = 0; k < W; ++k) {
    z[k] = acc[k];
    if (a.row_scale != nullptr) z[k] *= st * (k < count ? a.row_scale[i + k] : 0.0f);
    if (a.bias != nullptr) z[k] += bf16_to_f32(b[k]);
  }
  bf16_t zo[W], y[W];
#pragma unroll
  for (int k = 0; k < W; ++k) {
    zo[k] = f32_to_bf16(z[k]);
    float v = act_of(z[k], a.act);
    if (a.residual != nullptr) v += bf16_to_f32(r[k]);
    y[k] = f32_to_bf16(v);
  }
  if (count >= W) {
    if (a.preact != nullptr) __builtin_memcpy(a.preact + t * a.ldz + i, zo, sizeof zo);
    __builtin_memcpy(a.y + t * a.ldy + i, y, sizeof y);
  } else {
#pragma unroll
    for (int k = 0; k < W; ++k)
      if (k < count) {
        if (a.preact != nullptr) a.preact[t * a.ldz + i + k] = zo[k];
        a.y[t * a.ldy + i + k] = y[k];
      }
  }
}

// Tile `t` of mt x nt: strips of eight tile rows, in a strip column by column,
// so that the 32 workgroups of an XCD read 8 + 4 operand tiles a k step.
__device__ __forceinline__ void tile_at(uint32_t t, uint32_t mt, uint32_t nt, uint32_t& i, uint32_t& j) {
  const uint32_t strip = t / (8 * nt), u = t - strip * 8 * nt;
  const uint32_t r = min(8u, mt - strip * 8);
  i = strip * 8 + u % r;
  j = u / r;
}

// Scalar of a type's accumulator.
template <class T> struct Scalar { typedef float type; };
template <> struct Scalar<nt::I8> { typedef int32_t type; };

// Sums of 8-bit products lie in -127 128 n .. 128^2 n, n <= 2^17: the one that 32
// bits do not hold, 2^31 of (-128)^2 alone at n = 2^17, comes out as -2^31, which is
// none of them.
constexpr int64_t kWrapN = int64_t(1) << 17;
__device__ __forceinline__ float sum_f32(int32_t v) { return v == INT32_MIN ? 0x1p31f : (float)v; }
__device__ __forceinline__ float sum_f32(float v) { return v; }
__device__ __forceinline__ int32_t add(int32_t a, int32_t b) { return (int32_t)((uint32_t)a + (uint32_t)b); }
__device__ __forceinline__ float add(float a, float b) { return a + b; }

// TJ consecutive bf16 values of a row, as they lie in memory.
template <int TJ>
struct Piece {
  uint32_t w[TJ / 2];
  __device__ __forceinline__ float get(int j) const {
    return __builtin_bit_cast(float, j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
  }
  __device__ __forceinline__ void set(const float (&f)[TJ]) {
#pragma unroll
    for (int q = 0; q < TJ / 2; ++q)
      w[q] = (uint32_t)f32_to_bf16(f[2 * q]) | ((uint32_t)f32_to_bf16(f[2 * q + 1]) << 16);
  }
  // `count` of them exist (zeros beyond)
  __device__ __forceinline__ void load(const bf16_t* p, int count) {
    if (count >= TJ) {
      __builtin_memcpy(w, p, sizeof w);
    } else {
#pragma unroll
      for (int q = 0; q < TJ / 2; ++q) w[q] = 0;
#pragma unroll
      for (int j = 0; j < TJ - 1; ++j)
        if (j < count) w[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
    }
  }
  __device__ __forceinline__ void store(bf16_t* p, int count) const {
    if (count >= TJ) {
      __builtin_memcpy(p, w, sizeof w);
    } else {
#pragma unroll
      for (int j = 0; j < TJ - 1; ++j)
        if (j < count) p[j] = (bf16_t)(w[j >> 1] >> (16 * (j & 1)));
    }
  }
};

// Many tokens.  grid: tiles x splits.  P: null (one split), or splits x tokens
// x m sums.  Workgroups a compute unit: what its LDS holds.  256 x 256 tiles have
// the fewest operand bytes per product (1.36 us a pair, 2.0 POP/s in 8 bits for
// 4096 x 4096 -> 11008: 180 us, of which the last, partly filled round of 688
// tiles on 256 units costs a tenth); smaller ones fill the units where those
// are few (1021 x 1000 -> 777 bf16: 12.7 to 13.5 us, about 4 of them in the loop).
template <class T, int TI, int TJ, int SLOTS>
__global__ __launch_bounds__(nt::kThreads, ((TI + TJ) * SLOTS <= 20 ? 2 : 1)) void k_tile(
    LinearArgs a, uint32_t mt, uint32_t ntl, uint32_t splits, typename Scalar<T>::type* P) {
  typedef nt::Tile<T, TI, TJ, SLOTS> G;
  // (one object: beside a second one the compiler waits for every copy before each read)
  struct Shared {
    typename G::Ring ring;
    float xs[G::BM];  // the tile's row scales
  };
  __shared__ Shared all;
  typename G::Ring& sm = all.ring;
  float* xs = all.xs;
  const uint32_t tiles = mt * ntl;
  const uint32_t w = xcd_remap(blockIdx.x, gridDim.x);
  const uint32_t z = w / tiles;
  uint32_t ti, tj;
  tile_at(w - z * tiles, mt, ntl, ti, tj);
  const int64_t t0 = (int64_t)ti * G::BM, i0 = (int64_t)tj * G::BN;
  const nt::Rows A{(const char*)a.x + t0 * a.ldx * T::kBytes, (int)min((int64_t)G::BM, a.tokens - t0),
                   (uint32_t)(a.ldx * T::kBytes)};
  const nt::Rows B{(const char*)a.w + i0 * a.ldw * T::kBytes, (int)min((int64_t)G::BN, a.m - i0),
                   (uint32_t)(a.ldw * T::kBytes)};
  const int kbytes = (int)(a.n * T::kBytes), pairs = (kbytes + nt::kPair - 1) / nt::kPair;
  const int p0 = (int)((int64_t)pairs * z / splits), p1 = (int)((int64_t)pairs * (z + 1) / splits);
  const int64_t col = i0 + G::col_of(), row0 = t0 + G::row_of(0, 0);
  const int count = (int)min((int64_t)TJ, max((int64_t)0, a.m - col));
  const int rows = (int)min((int64_t)G::BM, a.tokens - row0);  // from row0 on (the lane's are 16 apart)
  float ws[TJ];
  Piece<TJ> bias, res[4], more[4];
  auto fetch = [&](int i) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (i * 16 + r < rows) more[r].load(a.residual + (row0 + i * 16 + r) * a.ldr + col, count);
  };
  const bool fused = P == nullptr && count > 0;
  if (fused) {
    if (a.row_scale != nullptr) {
#pragma unroll
      for (int j = 0; j < TJ; ++j) ws[j] = a.row_scale[min(col + j, a.m - 1)];
    }
    if (a.bias != nullptr) bias.load(a.bias + col, count);
    if (a.residual != nullptr) fetch(0);  // (all of these land during the loop)
  }
  typename G::Acc acc;
  G::zero(acc);
  static_assert(G::BM <= nt::kThreads, "a row a thread");
  if (a.x_scale != nullptr && (int)threadIdx.x < G::BM)
    xs[threadIdx.x] = (int)threadIdx.x < A.rows ? a.x_scale[t0 + threadIdx.x] : 0.0f;
  nt::Straight walk{A.p + p0 * nt::kPair, B.p + p0 * nt::kPair, kbytes - p0 * nt::kPair};
  G::loop(sm, A, B, p1 - p0, walk, acc);
  // The sums go through LDS (each lane its own 16-byte slots: no barrier, no
  // bank conflict) so that a short loop over four rows at a time serves all of
  // them: straight from the accumulators the epilogue of a 256 x 256 tile is 32
  // copies long and spills.  With one wave on a SIMD nothing hides a load, so a
  // lane's bias and scales are read once and the next rows' residual before
  // these rows' work; reading them row by row took 30 to 60 us a tile.
  typedef typename Scalar<T>::type S;
  // tile rows a phase, numbers of a piece of a row, pieces of a row
  constexpr int HI = TI < 4 ? TI : TI % 4 == 0 ? 4 : 3, PC = TJ % 4 == 0 ? 4 : 2, V = TJ / PC;
  typedef __attribute__((ext_vector_type(PC))) S Slot;
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
          Slot o;
#pragma unroll
          for (int e = 0; e < PC; ++e) o[e] = acc[h * HI + i][PC * v + e][r];
          stage[((i * 4 + r) * V + v) * nt::kThreads] = o;
        }
#pragma unroll 1
    for (int q = 0; q < HI; ++q) {
      const int i = h * HI + q;
      S s[4][TJ];
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const Slot o = stage[((q * 4 + r) * V + v) * nt::kThreads];
#pragma unroll
          for (int e = 0; e < PC; ++e) s[r][PC * v + e] = o[e];
        }
      if (fused) {
        if (a.residual != nullptr) {
#pragma unroll
          for (int r = 0; r < 4; ++r) res[r] = more[r];
          if (i + 1 < TI) fetch(i + 1);
        }
        float z[4][TJ];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int j = 0; j < TJ; ++j) z[r][j] = (float)s[r][j];
        if (std::is_same<T, nt::I8>::value && a.n == kWrapN) {  // (for any n it took 3 % of a prompt's time)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < TJ; ++j) z[r][j] = sum_f32(s[r][j]);
        }
        if (a.row_scale != nullptr) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(&xs[G::row_of(i, 0)]);
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < TJ; ++j) z[r][j] *= x[r] * ws[j];
        }
        if (a.bias != nullptr) {
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < TJ; ++j) z[r][j] += bias.get(j);
        }
        auto put = [&](bf16_t* p, int64_t ld) {
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            Piece<TJ> o;
            o.set(z[r]);
            if (i * 16 + r < rows) o.store(p + (row0 + i * 16 + r) * ld + col, count);
          }
        };
        if (a.preact != nullptr) put(a.preact, a.ldz);
        auto apply = [&](auto act) {
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < TJ; ++j) z[r][j] = act_as<decltype(act)::value>(z[r][j]);
        };
        if (a.act == kActRelu)
          apply(std::integral_constant<int, kActRelu>());
        else if (a.act == kActGelu)
          apply(std::integral_constant<int, kActGelu>());
        else if (a.act == kActSilu)
          apply(std::integral_constant<int, kActSilu>());
        if (a.residual != nullptr) {
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < TJ; ++j) z[r][j] += res[r].get(j);
        }
        put(a.y, a.ldy);
      } else if (P != nullptr) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (i * 16 + r < rows) {
            S* o = P + ((int64_t)z * a.tokens + row0 + i * 16 + r) * a.m + col;
            if (count == TJ) {
              __builtin_memcpy(o, s[r], sizeof s[r]);
            } else {
#pragma unroll
              for (int j = 0; j < TJ; ++j)
                if (j < count) o[j] = s[r][j];
            }
          }
      }
    }
  }
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

// 16 bytes of a row at byte k of `bytes`; zeros beyond.
template <int EB>
__device__ __forceinline__ u32x4 row_bytes(const char* row, int k, int bytes) {
  u32x4 v = {0, 0, 0, 0};
  if (k + 16 <= bytes) {
    __builtin_memcpy(&v, row + k, 16);
  } else {
    // the last, partial piece (whole elements)
#pragma unroll
    for (int e = 0; e < 16 / EB - 1; ++e)
      if (k + e * EB < bytes) {
        const uint32_t b = EB == 1 ? (uint32_t)(uint8_t)row[k + e] : (uint32_t)*(const uint16_t*)(row + k + e * EB);
        v[e * EB / 4] |= b << (8 * (e * EB % 4));
      }
  }
  return v;
}

// Few tokens.  One workgroup: 16 RW output rows; its waves take k in turn,
// 128 bytes a step: lane l holds bytes 32 (l / 16) .. + 31 of the step of row
// (token) l % 16, two matrix instructions' worth; which k a lane holds does not
// matter as long as both operands agree.  Accumulator element r of lane l:
// output row 4 (l / 16) + r, token l % 16.  Bound by reading w and, as a call is
// short, by the latency of its first bytes: one token, 4096 -> 11008 in 8 bits,
// 45 MB, in 12.8 to 14.3 us (3.2 to 3.5 TB/s).
template <class T, int NT, int RW, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_skinny(LinearArgs a) {
  typedef typename Scalar<T>::type S;
  __shared__ S sh[WAVES][RW * NT * 256];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t i0 = (int64_t)blockIdx.x * (16 * RW);
  const int bytes = (int)(a.n * T::kBytes), steps = (bytes + 127) / 128;
  const char* wr[RW];
#pragma unroll
  for (int r = 0; r < RW; ++r)  // rows beyond the matrix: its last one, not stored
    wr[r] = (const char*)a.w + min(i0 + r * 16 + (lane & 15), a.m - 1) * a.ldw * T::kBytes;
  const char* xr[NT];
  bool live[NT];
#pragma unroll
  for (int q = 0; q < NT; ++q) {
    const int64_t t = q * 16 + (lane & 15);
    live[q] = t < a.tokens;
    xr[q] = (const char*)a.x + (live[q] ? t : 0) * a.ldx * T::kBytes;
  }
  typename T::acc acc[RW][NT];
#pragma unroll
  for (int r = 0; r < RW; ++r)
#pragma unroll
    for (int q = 0; q < NT; ++q) acc[r][q] = typename T::acc{0, 0, 0, 0};
  const int kl = 32 * (lane >> 4);
  const int full = bytes / 128;
  auto products = [&](const u32x4 (&wv)[RW][2], const u32x4 (&xv)[NT][2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < RW; ++r)
#pragma unroll
        for (int q = 0; q < NT; ++q) acc[r][q] = T::mfma(wv[r][h], xv[q][h], acc[r][q]);
  };
  // U steps' loads go out before their products
  constexpr int U = RW + NT <= 2 ? 4 : RW + NT <= 5 ? 2 : 1;
  auto steps_at = [&](int s, auto count) {
    constexpr int C = decltype(count)::value;
    u32x4 wv[C][RW][2], xv[C][NT][2];
#pragma unroll
    for (int u = 0; u < C; ++u) {
      const int k = (s + u * WAVES) * 128 + kl;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int r = 0; r < RW; ++r) __builtin_memcpy(&wv[u][r][h], wr[r] + k + 16 * h, 16);
#pragma unroll
        for (int q = 0; q < NT; ++q) {
          xv[u][q][h] = u32x4{0, 0, 0, 0};
          if (live[q]) __builtin_memcpy(&xv[u][q][h], xr[q] + k + 16 * h, 16);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < C; ++u) products(wv[u], xv[u]);
  };
  int s = wave;
  for (; s + (U - 1) * WAVES < full; s += U * WAVES) steps_at(s, std::integral_constant<int, U>());
  for (; s < full; s += WAVES) steps_at(s, std::integral_constant<int, 1>());
  if (full < steps && full % WAVES == wave) {  // the last step: k ends inside it
    u32x4 wv[RW][2], xv[NT][2];
    const int k = full * 128 + kl;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int r = 0; r < RW; ++r) wv[r][h] = row_bytes<T::kBytes>(wr[r], k + 16 * h, bytes);
#pragma unroll
      for (int q = 0; q < NT; ++q)
        xv[q][h] = live[q] ? row_bytes<T::kBytes>(xr[q], k + 16 * h, bytes) : u32x4{0, 0, 0, 0};
    }
    products(wv, xv);
  }
#pragma unroll
  for (int r = 0; r < RW; ++r)
#pragma unroll
    for (int q = 0; q < NT; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e)  // token-major: 16 RW consecutive outputs of a token
        sh[wave][(q * 16 + (lane & 15)) * (16 * RW) + r * 16 + 4 * (lane >> 4) + e] = acc[r][q][e];
  __syncthreads();
  for (int o = threadIdx.x; o < RW * NT * 256; o += 64 * WAVES) {
    const int64_t t = o / (16 * RW), i = i0 + o % (16 * RW);
    if (t >= a.tokens || i >= a.m) continue;
    S v = sh[0][o];
#pragma unroll
    for (int k = 1; k < WAVES; ++k) v = add(v, sh[k][o]);
    const float f = sum_f32(v);
    finish<1>(a, t, i, &f, 1);
  }
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

// Q8: some job has codes for dy or z.  Eight columns lie within one group of them.
template <bool Q8>
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
    if (Q8 && a.dyq.q != nullptr) {
      float f[8];
      if (count > 0) {
        load_q8(a.dyq, row, col, count, f);
        v.set(f);
      }
    } else if (count > 0) {
      v = load_row(a.dy + row * a.lddy + col, count);
    }
    if ((a.z != nullptr || (Q8 && a.zq.q != nullptr)) && count > 0) {
      float f[8];
      if (Q8 && a.zq.q != nullptr) {
        load_q8(a.zq, row, col, count, f);
      } else {
        const Vec<bf16_t> z = load_row(a.z + row * a.ldz + col, count);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = z.get(k);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] = v.get(k) * act_slope(f[k], a.act);
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
  bool q8 = false;
  for (int k = 0; k < count; ++k) {
    const ActGradArgs& a = jobs[k];
    const int64_t gx = (a.cols + 63) / 64, gy = (a.rows + 63) / 64;
    if (a.rows <= 0 || a.cols <= 0 || gx * gy > 0x7fffffff ||
        (a.gt != nullptr && (a.ldgt % 8 != 0 || a.ldgt < a.rows || a.ldgt > gy * 64 || (uintptr_t)a.gt % 16 != 0)))
      return hipErrorInvalidValue;
    for (const Q8Rows* c : {&a.dyq, &a.zq}) {
      if (c->q == nullptr) continue;
      if (c->scale == nullptr || c->shift < kMinGroupShift || c->shift > kMaxGroupShift) return hipErrorInvalidValue;
      q8 = true;
    }
    total += gx * gy;
    if (total > 0x7fffffff) return hipErrorInvalidValue;
    q.job[k] = a;
    q.gx[k] = (uint32_t)gx;
    q.end[k] = (uint32_t)total;
  }
  for (int k = count; k < 3; ++k) q.end[k] = (uint32_t)total;
  if (q8)
    hipLaunchKernelGGL(k_turn<true>, dim3((uint32_t)total), dim3(256), 0, s, q);
  else
    hipLaunchKernelGGL(k_turn<false>, dim3((uint32_t)total), dim3(256), 0, s, q);
  return hipGetLastError();
}

}  // namespace ff
