// 8-bit checkpoints of activations: what a layer keeps of its input and its
// pre-activations for its gradient, in half the bytes of bf16.
//
//   a group's scale = max |x| / 127 (2^shift columns of a row), q = rint(127 x / max |x|),
//   and back: x' = q scale, off by at most half a scale.
//
// Both are bound by memory: 8192 x 8192 bf16 in 49 to 52 us (201 MB, 3.9 to 4.1 TB/s), and back, its
// codes still in the last-level cache, in 32.  A thread takes eight columns (16 bytes of
// bf16) of four pieces of the array at once, a group 2 to 64 neighbouring lanes, its largest
// magnitude one reduction over them.  A code hangs on which side of a half 127 x / max lies:
// x = max / 2 is 63.5 and must go to the even 64 whatever the division's last bit.  The
// quotient is taken as x (127 / max), off by at most 3 2^-24 127 < 2^-15, and where that
// lies within 2^-14 of a half it is taken again in 64 bits: 127 x is exact there, so a
// half stays one (the IEEE division of every element would cost 10 instructions each).
#include <math.h>

#include <algorithm>

#include "ff_layer_kernels.hpp"
#include "ff_q8.hpp"
#include "ff_vec.hpp"

namespace ff {
namespace {

// Eight elements of a row as they lie there, `count` of them in it, zeros after them.
template <class E>
struct Eight {
  static constexpr int N = Vec<E>::N;
  Vec<E> v[8 / N];
  __device__ __forceinline__ void load(const E* p, int count) {
#pragma unroll
    for (int h = 0; h < 8 / N; ++h) {
      v[h].w = u32x4{0, 0, 0, 0};
      if (count > h * N) v[h] = load_row(p + h * N, count - h * N);
    }
  }
  __device__ __forceinline__ float get(int i) const { return v[i / N].get(i % N); }
};
template <class E>
__device__ __forceinline__ void store8(E* p, int count, const float (&f)[8]) {
#pragma unroll
  for (int h = 0; h < 8 / Vec<E>::N; ++h) {
    constexpr int N = Vec<E>::N;
    if (count > h * N) {
      Vec<E> v;
      v.set(f + h * N);
      store_row(p + h * N, v, count - h * N);
    }
  }
}

__device__ __forceinline__ int code_of(float x, float big, float inv) {
  const float r = x * inv, near = rintf(r);
  if (__builtin_expect(fabsf(fabsf(r - near) - 0.5f) < 0x1p-14f, 0)) return (int)rint(127.0 * (double)x / (double)big);
  return (int)near;  // |r| <= 127 (1 + 2^-22): 127 at most
}

// A thread's piece: eight columns of a row.  `per_row` pieces a row, groups whole.
struct Pieces {
  int64_t total;
  uint32_t per_row;
};
// Piece `first + k` as row and column; first is the same for the workgroup's threads.
__device__ __forceinline__ void piece_at(const Pieces& p, int64_t first, uint32_t k, int64_t& row, int64_t& col) {
  const int64_t r = first / p.per_row;
  const uint32_t c = (uint32_t)(first - r * p.per_row) + k, more = c / p.per_row;
  row = r + more;
  col = (int64_t)(c - more * p.per_row) * 8;
}

constexpr int kUnits = 4;  // pieces a thread has in flight

template <class E>
__global__ __launch_bounds__(256) void k_checkpoint(CheckpointArgs a, Pieces p) {
  const int lanes = 1 << (a.shift - 3);  // of a group
  for (int64_t b = (int64_t)blockIdx.x * (256 * kUnits); b < p.total; b += (int64_t)gridDim.x * (256 * kUnits)) {
    Eight<E> x[kUnits];  // (as loaded: where a value is taken its load is waited for; 56 us so)
    int64_t row[kUnits], col[kUnits];
    int count[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const bool in = b + u * 256 + threadIdx.x < p.total;
      piece_at(p, b, u * 256 + threadIdx.x, row[u], col[u]);
      count[u] = in ? (int)min((int64_t)8, max((int64_t)0, a.cols - col[u])) : 0;
      x[u].load((const E*)a.x + row[u] * a.ldx + col[u], count[u]);
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = x[u].get(i);
      uint32_t bits = 0;  // of the largest magnitude; a NaN's are above all others
#pragma unroll
      for (int i = 0; i < 8; ++i) bits = max(bits, __float_as_uint(f[i]) & 0x7fffffffu);
      for (int d = 1; d < lanes; d <<= 1) bits = max(bits, (uint32_t)__shfl_xor((int)bits, d));
      const float big = __uint_as_float(bits);
      const bool finite = bits < 0x7f800000u, zero = big < 0x1p-118f;
      const float scale = !finite ? __uint_as_float(0x7fc00000u) : zero ? 0.0f : big / 127.0f;
      const float inv = !finite || zero ? 0.0f : 127.0f / big;
      if (count[u] <= 0) continue;
      uint32_t w[2] = {0, 0};
      if (inv != 0.0f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i / 4] |= ((uint32_t)code_of(f[i], big, inv) & 0xffu) << (8 * (i % 4));
      }
      int8_t* q = a.q + row[u] * a.ldq + col[u];
      if (count[u] == 8) {
        __builtin_memcpy(q, w, 8);
      } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
          if (i < count[u]) q[i] = (int8_t)(w[i / 4] >> (8 * (i % 4)));
      }
      if ((threadIdx.x & (lanes - 1)) == 0) a.scale[row[u] * a.lds + (col[u] >> a.shift)] = scale;
    }
  }
}

template <class E>
__global__ __launch_bounds__(256) void k_restore(CheckpointArgs a, Pieces p) {
  for (int64_t b = (int64_t)blockIdx.x * (256 * kUnits); b < p.total; b += (int64_t)gridDim.x * (256 * kUnits)) {
    uint32_t w[kUnits][2];
    float scale[kUnits];
    int64_t row[kUnits], col[kUnits];
    int count[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      piece_at(p, b, u * 256 + threadIdx.x, row[u], col[u]);
      count[u] = b + u * 256 + threadIdx.x < p.total ? (int)min((int64_t)8, a.cols - col[u]) : 0;
      if (count[u] > 0) {
        load_codes(a.q + row[u] * a.ldq + col[u], count[u], w[u]);
        scale[u] = a.scale[row[u] * a.lds + (col[u] >> a.shift)];
      }
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      if (count[u] <= 0) continue;
      float f[8];
      values_of(w[u], scale[u], f);
      store8((E*)a.x + row[u] * a.ldx + col[u], count[u], f);
    }
  }
}

bool fits(const CheckpointArgs& a) {
  return a.rows > 0 && a.cols > 0 && a.cols <= (int64_t(1) << 24) && a.shift >= kMinGroupShift &&
         a.shift <= kMaxGroupShift;
}
uint32_t blocks_for(const Pieces& p) {
  return (uint32_t)std::min<int64_t>((p.total + 256 * kUnits - 1) / (256 * kUnits), 1 << 20);
}

}  // namespace

hipError_t launch_checkpoint(const CheckpointArgs& a, bool bf16, hipStream_t s) {
  if (!fits(a)) return hipErrorInvalidValue;
  Pieces p;
  // groups whole, so that one never spans two workgroups' turns: 256 is a multiple of its lanes
  p.per_row = (uint32_t)(((a.cols + (int64_t(1) << a.shift) - 1) >> a.shift) << (a.shift - 3));
  p.total = a.rows * p.per_row;
  if (bf16)
    hipLaunchKernelGGL(k_checkpoint<bf16_t>, dim3(blocks_for(p)), dim3(256), 0, s, a, p);
  else
    hipLaunchKernelGGL(k_checkpoint<float>, dim3(blocks_for(p)), dim3(256), 0, s, a, p);
  return hipGetLastError();
}

hipError_t launch_restore(const CheckpointArgs& a, bool bf16, hipStream_t s) {
  if (!fits(a)) return hipErrorInvalidValue;
  Pieces p;
  p.per_row = (uint32_t)((a.cols + 7) / 8);
  p.total = a.rows * p.per_row;
  if (bf16)
    hipLaunchKernelGGL(k_restore<bf16_t>, dim3(blocks_for(p)), dim3(256), 0, s, a, p);
  else
    hipLaunchKernelGGL(k_restore<float>, dim3(blocks_for(p)), dim3(256), 0, s, a, p);
  return hipGetLastError();
}

}  // namespace ff
