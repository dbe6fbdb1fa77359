// A linear layer's tile and its few-token form, for one layer or for the layers of
// experts: what a workgroup does once it knows which rows and columns are its own.
#pragma once

#include <algorithm>
#include <type_traits>

#include "ff_layer_kernels.hpp"
#include "ff_tile_nt.hpp"
#include "ff_vec.hpp"

namespace ff {
namespace {

// sigmoid(x) = 1 / (1 + 2^(-x log2 e)) by the exponential and reciprocal
// instructions (one unit in the last place each; 0 below x = -87, 1 far out).  The
// argument's roundings, up to 3 2^-24 |x|, are relative errors of the exponential:
// 2^-19 of an activation at x = -10, 2^-16 where it ends, 1e-36; bf16's own is 2^-8.
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
// The workgroup's tile starts at row t0, column i0 and takes part z of k.  With
// order, row t of x is token order[t] / top's (32-bit byte offsets from x; rows that no
// token stands for are zeros).
template <class T, int TI, int TJ, int SLOTS>
struct LinearTile {
  typedef nt::Tile<T, TI, TJ, SLOTS> G;
  // (one object: beside a second one the compiler waits for every copy before each read)
  struct Shared {
    typename G::Ring ring;
    float xs[G::BM];  // the tile's row scales
  };
  static constexpr int kWaves = (TI + TJ) * SLOTS <= 20 ? 2 : 1;  // of a SIMD
  template <bool GATHER>
  static __device__ __forceinline__ void run(Shared& all, const LinearArgs& a, int64_t t0, int64_t i0, uint32_t z,
                                             uint32_t splits, typename Scalar<T>::type* P, const int32_t* order,
                                             int32_t top, int64_t x_rows);
};

template <class T, int TI, int TJ, int SLOTS>
template <bool GATHER>
__device__ __forceinline__ void LinearTile<T, TI, TJ, SLOTS>::run(Shared& all, const LinearArgs& a, int64_t t0,
                                                                  int64_t i0, uint32_t z, uint32_t splits,
                                                                  typename Scalar<T>::type* P, const int32_t* order,
                                                                  int32_t top, int64_t x_rows) {
  typename G::Ring& sm = all.ring;
  float* xs = all.xs;
  const nt::Rows A{(const char*)a.x + (GATHER ? 0 : t0 * a.ldx * T::kBytes), (int)min((int64_t)G::BM, a.tokens - t0),
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
  if constexpr (GATHER) {
    typename G::Lane lane = G::lane_of(A, B, threadIdx.x >> 6, threadIdx.x & 63);
#pragma unroll
    for (int q = 0; q < TI; ++q) {
      if (lane.a[q] == nt::kOutside) continue;
      const int32_t slot = order[t0 + (threadIdx.x >> 3) + 32 * q], t = slot / top;
      lane.a[q] = slot >= 0 && t < x_rows ? (uint32_t)t * A.ld + 16u * (uint32_t)lane.c : nt::kOutside;
    }
    G::loop(sm, lane, p1 - p0, walk, acc);
  } else {
    G::loop(sm, A, B, p1 - p0, walk, acc);
  }
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
// With order, row t of x is token order[t] / top's, as for the tiles.
template <class T, int NT, int RW, int WAVES>
using SkinnySums = typename Scalar<T>::type[WAVES][RW * NT * 256];
template <class T, int NT, int RW, int WAVES, bool GATHER>
__device__ __forceinline__ void skinny_run(SkinnySums<T, NT, RW, WAVES>& sh, const LinearArgs& a, int64_t i0,
                                           const int32_t* order, int32_t top, int64_t x_rows) {
  typedef typename Scalar<T>::type S;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
    int64_t row = live[q] ? t : 0;
    if (GATHER && live[q]) {
      const int32_t slot = order[t];
      row = slot / top;
      live[q] = slot >= 0 && row < x_rows;
      row = live[q] ? row : 0;
    }
    xr[q] = (const char*)a.x + row * a.ldx * T::kBytes;
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

}  // namespace
}  // namespace ff
