// 16-byte pieces of rows that need not start 16-byte aligned (odd widths,
// slices): global loads and stores of any alignment are one instruction on
// gfx950, a misaligned one only touches one more cache line.
#pragma once

#include "ff_common.hpp"

namespace ff {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

template <class E> struct Vec;
template <> struct Vec<bf16_t> {
  static constexpr int N = 8;
  u32x4 w;
  __device__ __forceinline__ bf16_t bits(int i) const { return (bf16_t)(w[i >> 1] >> (16 * (i & 1))); }
  __device__ __forceinline__ void set_bits(int i, bf16_t b) {
    w[i >> 1] = i & 1 ? (w[i >> 1] & 0xffffu) | ((uint32_t)b << 16) : (w[i >> 1] & 0xffff0000u) | b;
  }
  __device__ __forceinline__ float get(int i) const {
    return __builtin_bit_cast(float, i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
  }
  __device__ __forceinline__ void set(const float* f) {  // rounded to nearest even
#pragma unroll
    for (int q = 0; q < 4; ++q) w[q] = (uint32_t)f32_to_bf16(f[2 * q]) | ((uint32_t)f32_to_bf16(f[2 * q + 1]) << 16);
  }
};
template <> struct Vec<float> {
  static constexpr int N = 4;
  u32x4 w;
  __device__ __forceinline__ uint32_t bits(int i) const { return w[i]; }
  __device__ __forceinline__ void set_bits(int i, uint32_t b) { w[i] = b; }
  __device__ __forceinline__ float get(int i) const {
    const uint32_t b = w[i];  // (a bit cast of the vector's element itself reads element 0)
    return __builtin_bit_cast(float, b);
  }
  __device__ __forceinline__ void set(const float* f) {
#pragma unroll
    for (int q = 0; q < 4; ++q) w[q] = __builtin_bit_cast(uint32_t, f[q]);
  }
};

// `count` elements from p on (N or more: all), zeros after them.
template <class E>
__device__ __forceinline__ Vec<E> load_row(const E* p, int64_t count) {
  Vec<E> v;
  if (count >= Vec<E>::N) {
    __builtin_memcpy(&v.w, p, 16);
  } else {
    v.w = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < Vec<E>::N - 1; ++i)
      if (i < count) {
        decltype(v.bits(0)) b;
        __builtin_memcpy(&b, p + i, sizeof(E));
        v.set_bits(i, b);
      }
  }
  return v;
}
template <class E>
__device__ __forceinline__ void store_row(E* p, const Vec<E>& v, int64_t count) {
  if (count >= Vec<E>::N) {
    __builtin_memcpy(p, &v.w, 16);
  } else {
#pragma unroll
    for (int i = 0; i < Vec<E>::N - 1; ++i)
      if (i < count) {
        const auto b = v.bits(i);
        __builtin_memcpy(p + i, &b, sizeof(E));
      }
  }
}

}  // namespace ff
