// Shared device-side definitions of the FlipFlop engine (gfx950 / CDNA4).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ff {

// Vector types of the matrix-core builtins.
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef uint16_t bf16_t;  // bf16 bit pattern in memory

// Device status block shared by every kernel of one handle.
//   st[0]: 0 = healthy; otherwise the 1-based global iteration at which a
//          factor to be inverted was not positive definite.
//   st[1]: side that failed (1 = A, 2 = B).
//   st[2]: 0-based pivot index of the first failing pivot.
//   st[3]: 0, or the 1-based global iteration after which the relative
//          change of A (x) B fell to the caller's tolerance.
// Every kernel that belongs to the iteration returns at once when st[0] or
// st[3] is set, so that the factors of the last completed iteration stay
// intact.
__device__ __forceinline__ bool ff_halted(const int* st) {
  return st != nullptr && (__builtin_nontemporal_load(st) | __builtin_nontemporal_load(st + 3)) != 0;
}

__device__ __forceinline__ bf16_t f32_to_bf16(float x) {
  __bf16 h = (__bf16)x;  // round to nearest even (v_cvt_pk_bf16_f32)
  return __builtin_bit_cast(bf16_t, h);
}

__device__ __forceinline__ float bf16_to_f32(bf16_t b) {
  return __builtin_bit_cast(float, (uint32_t)b << 16);
}

template <typename T> struct Elem;
template <> struct Elem<float> {
  __device__ static float from_f32(float x) { return x; }
  __device__ static float to_f32(float x) { return x; }
};
template <> struct Elem<bf16_t> {
  __device__ static bf16_t from_f32(float x) { return f32_to_bf16(x); }
  __device__ static float to_f32(bf16_t x) { return bf16_to_f32(x); }
};

// Workgroups of one launch are spread round-robin over the 8 XCDs (each with
// its own L2).  Remap the hardware id so that consecutive logical ids run on
// the same XCD; a bijection for any grid size.
__device__ __forceinline__ uint32_t xcd_remap(uint32_t w, uint32_t total) {
  const uint32_t q = total >> 3, r = total & 7u;
  const uint32_t x = w & 7u, local = w >> 3;
  const uint32_t start = x < r ? x * (q + 1) : r * (q + 1) + (x - r) * q;
  return start + local;
}

// Upper-triangle tile index -> (ti, tj), ti <= tj, row-major over the triangle.
__device__ __forceinline__ void upper_tile(uint32_t idx, uint32_t T, uint32_t& ti, uint32_t& tj) {
  uint32_t i = 0, rowlen = T;
  while (idx >= rowlen) {
    idx -= rowlen;
    ++i;
    --rowlen;
  }
  ti = i;
  tj = i + idx;
}

// Order in which the workgroups of one k split visit the upper tiles: tile
// rows and columns are grouped in fours; the 4 x 4 groups are visited
// column by column (group Q = 0, 1, ..., and in group column Q the groups
// P = 0..Q), the tiles of an off-diagonal group column-major and those of a
// diagonal group row-major over its upper triangle.  Consecutive workgroups
// share an XCD (and its L2); in this order a window of them reads fewer
// distinct tile rows than in the row-major order (12% fewer L2 misses and
// 3% less time on the 4096-wide symmetric product).
constexpr uint32_t TGRP = 4;
__device__ __forceinline__ void grouped_tile(uint32_t idx, uint32_t T, uint32_t& ti, uint32_t& tj) {
  for (uint32_t Q = 0, q0 = 0; q0 < T; ++Q, q0 += TGRP) {
    const uint32_t sq = min(TGRP, T - q0);          // tiles in this group column
    const uint32_t off = Q * TGRP * sq;             // its off-diagonal groups (all full height)
    const uint32_t cnt = off + sq * (sq + 1) / 2;
    if (idx < cnt) {
      if (idx < off) {
        const uint32_t P = idx / (TGRP * sq), r = idx % (TGRP * sq);
        ti = P * TGRP + r % TGRP;
        tj = q0 + r / TGRP;
      } else {
        uint32_t a, b;
        upper_tile(idx - off, sq, a, b);
        ti = q0 + a;
        tj = q0 + b;
      }
      return;
    }
    idx -= cnt;
  }
  ti = tj = 0;
}

}  // namespace ff
