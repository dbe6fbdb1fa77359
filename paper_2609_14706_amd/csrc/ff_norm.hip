// Root-mean-square norm of rows with the residual's addition, its output in
// the rows' type or in 8 bits with a scale for each row, and its gradient.
//
//   s = x + r,  i = 1 / sqrt(mean_j s_j^2 + eps),  y_j = s_j i w_j
//   8 bits:  h_j = y_j alpha_j,  scale = max_j |h_j| / 127,  q_j = rint(h_j / scale)
//   gradient, with u = dy w:  ds = i (u - s i^2 mean_j(u_j s_j)) (+ dsum),
//             dw_j = sum_t dy_tj s_tj i_t
//
// Both are bound by memory: every row is read once, held in registers (fp32)
// through its reductions and written once.  A row takes one wave (up to two
// vectors of 16 bytes a lane) or a workgroup of 128 to 1024 threads; rows too
// long for registers (above 32768 bf16, 16384 fp32) are read again for each
// pass (k_norm_long, k_norm_grad_long).  8192 x 8192 bf16 with residual to 8
// bits: 99 us, 4.7 TB/s where a large copy reaches 5.1; gradient of 8191 x 4096:
// 53 us (5.1 TB/s) and 5 us for the sums of dw.
// All sums are fp32, in an order fixed by the sizes.  A row whose squares leave
// fp32's range (mean s^2 + eps not in 2^-100 .. 2^128) is summed again with s and
// eps scaled by a power of two.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "ff_layer_kernels.hpp"
#include "ff_vec.hpp"

namespace ff {
namespace {

template <class E>
__device__ __forceinline__ float f32(E x) { return Elem<E>::to_f32(x); }

// Sum over the THR threads of a row; the result in all of them.  red: a slot
// per wave.  Two barriers when the row spans waves (the slots are free again).
template <int THR, class Op>
__device__ __forceinline__ float row_reduce(float v, float* red, Op op) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = op(v, __shfl_xor(v, d));
  if (THR > 64) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) red[wave] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int k = 1; k < THR / 64; ++k) v = op(v, red[k]);
    __syncthreads();
  }
  return v;
}
struct Add {
  __device__ float operator()(float a, float b) const { return a + b; }
};
// Whether fp32 holds m = mean s^2 + eps and the squares that matter in it; if
// not, the factor of s with which it does, kUp or kDown (a row of NaN or infinities
// gets one too, to no effect), and eps with it.  s from 2^-149 on to 2^-43 becomes
// 2^-49 .. 2^57, from 2^57 on 2^-23 .. 2^48.
constexpr float kUp = 0x1p100f, kDown = 0x1p-80f;
__device__ __forceinline__ bool in_range(float m) { return m >= 0x1p-100f && m < INFINITY; }
struct One {};
__device__ __forceinline__ float operator*(float v, One) { return v; }
// A value that every lane of the wave holds, as one for all of them.
__device__ __forceinline__ float uniform(float v) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v)));
}

// Largest bit pattern: of magnitudes the largest, and a NaN above them all.
struct MaxBits {
  __device__ float operator()(float a, float b) const {
    return __float_as_uint(a) > __float_as_uint(b) ? a : b;
  }
};

// The scale of a row whose largest |h| is `big` and the factor that takes h to
// its code.  A row that is not finite gets a NaN scale and zero codes; one too
// small for a normal scale (zeros among them) counts as zeros.
__device__ __forceinline__ void row_scale(float big, float& scale, float& inv) {
  if (!(__float_as_uint(big) < 0x7f800000u)) {
    scale = __uint_as_float(0x7fc00000u);
    inv = 0.0f;
  } else if (big < 0x1p-118f) {
    scale = inv = 0.0f;
  } else {
    scale = big / 127.0f;
    inv = 127.0f / big;
  }
}
__device__ __forceinline__ int code_of(float h, float inv) {
  // finite h: |h inv| <= 127 (1 + 2^-22), which rounds to at most 127
  return inv == 0.0f ? 0 : (int)rintf(h * inv);
}

// N codes (8 or 4 bytes) of one 16-byte vector of E; `count` of them exist.
template <int N>
__device__ __forceinline__ void store_codes(int8_t* p, const float (&h)[N], float inv, int64_t count) {
  uint32_t w[N / 4];
#pragma unroll
  for (int q = 0; q < N / 4; ++q) {
    w[q] = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[q] |= ((uint32_t)code_of(h[4 * q + i], inv) & 0xffu) << (8 * i);
  }
  if (count >= N) {
    __builtin_memcpy(p, w, N);
  } else {
#pragma unroll
    for (int i = 0; i < N - 1; ++i)
      if (i < count) p[i] = (int8_t)(w[i / 4] >> (8 * (i % 4)));
  }
}

// Threads of a workgroup of rows that take THR each: a row, or four of a wave.
constexpr int block_of(int thr) { return thr == 64 ? 256 : thr; }

// THR threads a row, VPT vectors a thread.  Q8: codes and scales; otherwise y.
template <class E, int THR, int VPT, bool Q8>
__global__ __launch_bounds__(block_of(THR)) void k_norm(NormArgs a) {
  constexpr int N = Vec<E>::N, RPB = block_of(THR) / THR;
  __shared__ float red[16];
  const int t = threadIdx.x % THR;
  for (int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / THR; row < a.rows;
       row += (int64_t)gridDim.x * RPB) {
    const E* x = (const E*)a.x + row * a.ldx;
    const E* r = (const E*)a.residual + row * a.ldr;
    float s[VPT][N];
    Vec<E> vw[VPT];
    {
      Vec<E> vx[VPT], vr[VPT];
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        const int64_t j = (int64_t)(k * THR + t) * N, left = a.cols - j;
        if (left > 0) {
          vx[k] = load_row(x + j, left);
          if (a.residual != nullptr) vr[k] = load_row(r + j, left);
          if (a.weight != nullptr) vw[k] = load_row((const E*)a.weight + j, left);
        } else {
          vx[k].w = vr[k].w = vw[k].w = u32x4{0, 0, 0, 0};
        }
      }
#pragma unroll
      for (int k = 0; k < VPT; ++k)
#pragma unroll
        for (int i = 0; i < N; ++i) {
          s[k][i] = vx[k].get(i);
          if (a.residual != nullptr) s[k][i] += vr[k].get(i);
        }
    }
    if (a.sum != nullptr) {
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        const int64_t j = (int64_t)(k * THR + t) * N, left = a.cols - j;
        if (left > 0) {
          Vec<E> o;
          o.set(s[k]);
          store_row((E*)a.sum + row * a.ldsum + j, o, left);
        }
      }
    }
    float inv_rms = 1.0f;
    if (a.normalise) {
      float eps = a.eps.plain;
#pragma unroll 1
      for (int pass = 0;; ++pass) {  // (every thread of a row takes the same passes)
        float ss = 0.0f;
#pragma unroll
        for (int k = 0; k < VPT; ++k)
#pragma unroll
          for (int i = 0; i < N; ++i) ss += s[k][i] * s[k][i];
        const float m = uniform(row_reduce<THR>(ss, red, Add()) / (float)a.cols + eps);
        inv_rms = 1.0f / sqrtf(m);
        if (pass == 1 || in_range(m)) break;
        const float f = m < 1.0f ? kUp : kDown;
        eps = m < 1.0f ? a.eps.up : a.eps.down;
#pragma unroll
        for (int k = 0; k < VPT; ++k)
#pragma unroll
          for (int i = 0; i < N; ++i) s[k][i] *= f;
      }
    }
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        s[k][i] *= inv_rms;
        if (a.weight != nullptr) s[k][i] *= vw[k].get(i);
      }
      if (Q8 && a.col_scale != nullptr) {
        const int64_t j = (int64_t)(k * THR + t) * N, left = a.cols - j;
#pragma unroll
        for (int h = 0; h < N / 4; ++h) {
          const Vec<float> c = left > 4 * h ? load_row(a.col_scale + j + 4 * h, left - 4 * h) : Vec<float>{};
#pragma unroll
          for (int i = 0; i < 4; ++i) s[k][4 * h + i] *= c.get(i);
        }
      }
    }
    if (!Q8) {
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        const int64_t j = (int64_t)(k * THR + t) * N, left = a.cols - j;
        if (left > 0) {
          Vec<E> o;
          o.set(s[k]);
          store_row((E*)a.y + row * a.ldy + j, o, left);
        }
      }
    } else {
      float big = 0.0f;
#pragma unroll
      for (int k = 0; k < VPT; ++k)
#pragma unroll
        for (int i = 0; i < N; ++i) {
          // (elements beyond the row may be 0 inf = NaN here)
          const float h = (int64_t)(k * THR + t) * N + i < a.cols ? fabsf(s[k][i]) : 0.0f;
          big = MaxBits()(big, h);
        }
      big = row_reduce<THR>(big, red, MaxBits());
      float scale, inv;
      row_scale(big, scale, inv);
      if (t == 0) a.q_scale[row] = scale;
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        const int64_t j = (int64_t)(k * THR + t) * N, left = a.cols - j;
        if (left > 0) store_codes<N>(a.q + row * a.ldq + j, s[k], inv, left);
      }
    }
  }
}

// Rows of any length: one workgroup a row, read again in each pass.
template <class E, bool Q8>
__global__ __launch_bounds__(1024) void k_norm_long(NormArgs a) {
  __shared__ float red[16];
  const E* W = (const E*)a.weight;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const E* x = (const E*)a.x + row * a.ldx;
    const E* r = a.residual != nullptr ? (const E*)a.residual + row * a.ldr : nullptr;
    auto at = [&](int64_t j) { return f32<E>(x[j]) + (r != nullptr ? f32<E>(r[j]) : 0.0f); };
    float inv_rms = 1.0f, f = 1.0f;
    if (a.normalise) {
      float eps = a.eps.plain;
      for (int pass = 0;; ++pass) {
        float ss = 0.0f;
        for (int64_t j = threadIdx.x; j < a.cols; j += 1024) ss += (at(j) * f) * (at(j) * f);
        const float m = uniform(row_reduce<1024>(ss, red, Add()) / (float)a.cols + eps);
        inv_rms = 1.0f / sqrtf(m);
        if (pass == 1 || in_range(m)) break;
        f = m < 1.0f ? kUp : kDown;
        eps = m < 1.0f ? a.eps.up : a.eps.down;
      }
    }
    auto h = [&](int64_t j) {
      float c = W != nullptr ? f32<E>(W[j]) : 1.0f;
      if (Q8 && a.col_scale != nullptr) c *= a.col_scale[j];
      return at(j) * f * inv_rms * c;
    };
    float scale = 0.0f, inv = 0.0f;
    if (Q8) {
      float big = 0.0f;
      for (int64_t j = threadIdx.x; j < a.cols; j += 1024) big = MaxBits()(big, fabsf(h(j)));
      big = row_reduce<1024>(big, red, MaxBits());
      row_scale(big, scale, inv);
      if (threadIdx.x == 0) a.q_scale[row] = scale;
    }
    for (int64_t j = threadIdx.x; j < a.cols; j += 1024) {
      const float v = h(j), s = at(j);  // sum and y may be x's own rows: read first
      if (a.sum != nullptr) ((E*)a.sum)[row * a.ldsum + j] = Elem<E>::from_f32(s);
      if (Q8)
        a.q[row * a.ldq + j] = (int8_t)code_of(v, inv);
      else
        ((E*)a.y)[row * a.ldy + j] = Elem<E>::from_f32(v);
    }
  }
}

// Gradient: as k_norm, with the columns' share of dw summed over the
// workgroup's rows and left in part[workgroup][column].  Rows that need scaling
// are left until after up to 63 others: taken at once they cost all rows registers
// (1024 x 32768 bf16: 188 us, 100 so).
template <class E, int THR, int VPT>
__global__ __launch_bounds__(block_of(THR)) void k_norm_grad(NormGradArgs a) {
  constexpr int N = Vec<E>::N, RPB = block_of(THR) / THR;
  __shared__ float red[32];
  __shared__ float share[RPB > 1 ? RPB * 64 * VPT * N : 1];
  const int t = threadIdx.x % THR, cols = (int)a.cols;
  float dw[VPT][N];
  Vec<E> vw[VPT];
#pragma unroll
  for (int k = 0; k < VPT; ++k) {
    const int j = (k * THR + t) * N, left = cols - j;
    if (a.weight != nullptr && left > 0) vw[k] = load_row((const E*)a.weight + j, left);
#pragma unroll
    for (int i = 0; i < N; ++i) dw[k][i] = 0.0f;
  }
  auto w = [&](int k, int i) { return a.weight != nullptr ? vw[k].get(i) : 1.0f; };
  // One row; false, and nothing done, where it has to be scaled (the same for every
  // thread of a row)
  auto plain_row = [&](int64_t row) {
    Vec<E> vs[VPT], vd[VPT], vt[VPT];
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int j = (k * THR + t) * N, left = cols - j;
      if (left > 0) {
        vs[k] = load_row((const E*)a.s + row * a.lds + (uint32_t)j, left);
        vd[k] = load_row((const E*)a.dy + row * a.lddy + (uint32_t)j, left);
        if (a.dsum != nullptr) vt[k] = load_row((const E*)a.dsum + row * a.lddsum + (uint32_t)j, left);
      }
    }
    float ss = 0.0f, us = 0.0f;
#pragma unroll
    for (int k = 0; k < VPT; ++k)
      if (cols - (k * THR + t) * N > 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float s = vs[k].get(i);
          ss += s * s;
          us += vd[k].get(i) * w(k, i) * s;
        }
      }
    ss = row_reduce<THR>(ss, red, Add());
    us = row_reduce<THR>(us, red + 16, Add());
    // (dsum's loads have landed by now; said here, or the compiler waits at the next row's
    // start for whatever is on its way, this one's stores too: 4096 x 8192 53 us, 49 so)
    __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));  // vmcnt(0)
    const float m = ss / (float)a.cols + a.eps.plain;
    if (__builtin_expect(!in_range(m), 0)) return false;
    const float i1 = 1.0f / sqrtf(m);
    const float proj = us / (float)a.cols * i1 * i1;
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int j = (k * THR + t) * N, left = cols - j;
      if (left > 0) {
        float g[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float s = vs[k].get(i), d = vd[k].get(i);
          dw[k][i] += d * s * i1;
          g[i] = i1 * (d * w(k, i) - s * proj);
          if (a.dsum != nullptr) g[i] += vt[k].get(i);
        }
        Vec<E> o;
        o.set(g);
        store_row((E*)a.dx + row * a.lddx + (uint32_t)j, o, left);
      }
    }
    return true;
  };
  // One that has to be scaled: read again for each pass, a vector at a time
  auto scaled_row = [&](int64_t row) {
    const E* const s_row = (const E*)a.s + row * a.lds;
    const E* const d_row = (const E*)a.dy + row * a.lddy;
    float f = 1.0f, us = 0.0f, m = 0.0f;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
      float ss = 0.0f;
      us = 0.0f;
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        const int j = (k * THR + t) * N, left = cols - j;
        if (left > 0) {
          const Vec<E> vs = load_row(s_row + (uint32_t)j, left), vd = load_row(d_row + (uint32_t)j, left);
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const float s = vs.get(i) * f;
            ss += s * s;
            us += vd.get(i) * w(k, i) * s;
          }
        }
        __builtin_amdgcn_sched_barrier(0);  // (the next vector's loads stay behind)
      }
      ss = row_reduce<THR>(ss, red, Add());
      us = row_reduce<THR>(us, red + 16, Add());
      m = ss / (float)a.cols + (f == 1.0f ? a.eps.plain : f == kUp ? a.eps.up : a.eps.down);
      if (pass == 0) f = m < 1.0f ? kUp : kDown;
    }
    const float i1 = 1.0f / sqrtf(m);
    const float proj = us / (float)a.cols * i1 * i1;
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int j = (k * THR + t) * N, left = cols - j;
      if (left > 0) {
        const Vec<E> vs = load_row(s_row + (uint32_t)j, left), vd = load_row(d_row + (uint32_t)j, left);
        float g[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float s = vs.get(i) * f, d = vd.get(i);
          dw[k][i] += d * s * i1;
          g[i] = i1 * (d * w(k, i) - s * proj) * f;
        }
        if (a.dsum != nullptr) {
          const Vec<E> vt = load_row((const E*)a.dsum + row * a.lddsum + (uint32_t)j, left);
#pragma unroll
          for (int i = 0; i < N; ++i) g[i] += vt.get(i);
        }
        Vec<E> o;
        o.set(g);
        store_row((E*)a.dx + row * a.lddx + (uint32_t)j, o, left);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  const int64_t step = (int64_t)gridDim.x * RPB;
  const int wave = RPB > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;  // whose row it is
  for (int64_t row0 = (int64_t)blockIdx.x * RPB + wave; row0 < a.rows; row0 += 64 * step) {
    uint64_t later = 0;  // (dx may be s itself: a row that is done is not looked at again)
    int64_t row = row0;
    for (int i = 0; i < 64 && row < a.rows; ++i, row += step)
      if (!plain_row(row)) later |= uint64_t(1) << i;
    while (__builtin_expect(later != 0, 0)) {
      scaled_row(row0 + __builtin_ctzll(later) * step);
      later &= later - 1;
    }
  }
  if (a.part == nullptr) return;
  float* part = a.part + (int64_t)blockIdx.x * a.cols;
  if (RPB > 1) {
#pragma unroll
    for (int k = 0; k < VPT; ++k)
#pragma unroll
      for (int i = 0; i < N; ++i) share[(threadIdx.x / THR) * (64 * VPT * N) + (k * THR + t) * N + i] = dw[k][i];
    __syncthreads();
    for (int j = threadIdx.x; j < a.cols; j += 256) {
      float v = 0.0f;
#pragma unroll
      for (int b = 0; b < RPB; ++b) v += share[b * (64 * VPT * N) + j];
      part[j] = v;
    }
  } else {
#pragma unroll
    for (int k = 0; k < VPT; ++k)
#pragma unroll
      for (int i = 0; i < N; ++i)
        if ((int64_t)(k * THR + t) * N + i < a.cols) part[(int64_t)(k * THR + t) * N + i] = dw[k][i];
  }
}

template <class E>
__global__ __launch_bounds__(1024) void k_norm_grad_long(NormGradArgs a) {
  __shared__ float red[32];
  const E* W = (const E*)a.weight;
  float* part = a.part != nullptr ? a.part + (int64_t)blockIdx.x * a.cols : nullptr;
  if (part != nullptr)
    for (int64_t j = threadIdx.x; j < a.cols; j += 1024) part[j] = 0.0f;  // this thread's own columns
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const E* s = (const E*)a.s + row * a.lds;
    const E* dy = (const E*)a.dy + row * a.lddy;
    const E* ds = a.dsum != nullptr ? (const E*)a.dsum + row * a.lddsum : nullptr;
    // the row with s scaled by f; returns mean s^2 + eps, and stores where it is in
    // range or f is not one
    auto turn = [&](auto f, float eps) {
      float ss = 0.0f, us = 0.0f;
      for (int64_t j = threadIdx.x; j < a.cols; j += 1024) {
        const float v = f32<E>(s[j]) * f;
        ss += v * v;
        us += f32<E>(dy[j]) * (W != nullptr ? f32<E>(W[j]) : 1.0f) * v;
      }
      ss = row_reduce<1024>(ss, red, Add());
      us = row_reduce<1024>(us, red + 16, Add());
      const float m = uniform(ss / (float)a.cols + eps), i1 = 1.0f / sqrtf(m);
      if (std::is_same<decltype(f), One>::value && !in_range(m)) return m;
      const float proj = us / (float)a.cols * i1 * i1;
      for (int64_t j = threadIdx.x; j < a.cols; j += 1024) {
        const float v = f32<E>(s[j]) * f, d = f32<E>(dy[j]);
        if (part != nullptr) part[j] += d * v * i1;
        float g = i1 * (d * (W != nullptr ? f32<E>(W[j]) : 1.0f) - v * proj) * f;
        if (ds != nullptr) g += f32<E>(ds[j]);
        ((E*)a.dx)[row * a.lddx + j] = Elem<E>::from_f32(g);
      }
      return m;
    };
    const float m = turn(One(), a.eps.plain);
    if (!in_range(m)) turn(m < 1.0f ? kUp : kDown, m < 1.0f ? a.eps.up : a.eps.down);
  }
}

// out[j] = sum_p part[p][j]: 32 columns x 32 groups of rows a workgroup.
template <class E>
__global__ __launch_bounds__(1024) void k_col_sums(const float* part, int64_t rows, int64_t cols, E* out) {
  __shared__ float sh[32][33];
  const int c = threadIdx.x & 31, g = threadIdx.x >> 5;
  const int64_t j = (int64_t)blockIdx.x * 32 + c;
  float v = 0.0f;
  if (j < cols)
    for (int64_t r = g; r < rows; r += 32) v += part[r * cols + j];
  sh[g][c] = v;
  __syncthreads();
  if (g == 0 && j < cols) {
#pragma unroll
    for (int k = 1; k < 32; ++k) v += sh[k][c];
    out[j] = Elem<E>::from_f32(v);
  }
}

// Threads and vectors a thread for rows of `cols`: one or two vectors a thread
// up to 1024 vectors (8192 x 8192 to 8 bits: 512 x 2 99 us, 256 x 4 108 us), four beyond.
// Few rows (under 512: not one a compute unit twice over) go to 1024 threads,
// which hold a row in one vector each: latency is what counts there.
struct Shape {
  int thr, vpt;
};
Shape norm_shape(int64_t rows, int64_t cols, int elems) {
  const int64_t nv = (cols + elems - 1) / elems;
  if (nv <= 64) return {64, 1};
  if (rows < 512 && nv <= 1024 && nv > 128) return {1024, 1};
  if (nv <= 128) return {64, 2};
  if (nv <= 256) return {128, 2};
  if (nv <= 512) return {256, 2};
  if (nv <= 1024) return {512, 2};
  if (nv <= 2048) return {512, 4};
  if (nv <= 4096) return {1024, 4};
  return {0, 0};
}

template <class E, bool Q8>
hipError_t norm_for(const NormArgs& a, hipStream_t s) {
  const Shape sh = norm_shape(a.rows, a.cols, Vec<E>::N);
  const int rpb = sh.thr == 64 ? 4 : 1;
  const int64_t blocks = std::min<int64_t>((a.rows + rpb - 1) / rpb, 4096);
  const dim3 grid((uint32_t)blocks);
#define FF_CASE(T, V)                                                                          \
  if (sh.thr == T && sh.vpt == V) {                                                            \
    hipLaunchKernelGGL((k_norm<E, T, V, Q8>), grid, dim3(block_of(T)), 0, s, a);               \
    return hipGetLastError();                                                                  \
  }
  FF_CASE(64, 1) FF_CASE(64, 2) FF_CASE(128, 2) FF_CASE(256, 2) FF_CASE(512, 2) FF_CASE(512, 4)
  FF_CASE(1024, 1) FF_CASE(1024, 4)
#undef FF_CASE
  hipLaunchKernelGGL((k_norm_long<E, Q8>), dim3((uint32_t)std::min<int64_t>(a.rows, 512)), dim3(1024), 0, s, a);
  return hipGetLastError();
}

template <class E>
hipError_t grad_for(const NormGradArgs& a, hipStream_t s) {
  const Shape sh = norm_shape(a.rows, a.cols, Vec<E>::N);
  const dim3 grid((uint32_t)norm_grad_parts(a.rows));
#define FF_CASE(T, V)                                                                          \
  if (sh.thr == T && sh.vpt == V) {                                                            \
    hipLaunchKernelGGL((k_norm_grad<E, T, V>), grid, dim3(block_of(T)), 0, s, a);              \
  } else
  FF_CASE(64, 1) FF_CASE(64, 2) FF_CASE(128, 2) FF_CASE(256, 2) FF_CASE(512, 2) FF_CASE(512, 4)
  FF_CASE(1024, 1) FF_CASE(1024, 4)
#undef FF_CASE
  hipLaunchKernelGGL((k_norm_grad_long<E>), grid, dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace

// Workgroups of the gradient, each with a row of partial sums of dw: two a
// compute unit; few rows take one, their partial sums weigh as much as they do
// (2048 x 16384 bf16: 82 us with 512, 67 us with 256; 8191 x 4096: 60 and 84).
int64_t norm_grad_parts(int64_t rows) { return std::min<int64_t>(rows, rows < 4096 ? 256 : 512); }

Eps eps_of(double eps) {
  // (positive where eps is: rows of zeros stay zeros)
  auto at = [&](double f) { return eps > 0.0 ? std::max((float)(eps * f * f), 0x1p-149f) : 0.0f; };
  return {at(1.0), at(kUp), at(kDown)};
}

hipError_t launch_norm(const NormArgs& a, bool bf16, hipStream_t s) {
  if (a.rows <= 0 || a.cols <= 0) return hipErrorInvalidValue;
  if (bf16) return a.q != nullptr ? norm_for<bf16_t, true>(a, s) : norm_for<bf16_t, false>(a, s);
  return a.q != nullptr ? norm_for<float, true>(a, s) : norm_for<float, false>(a, s);
}

hipError_t launch_norm_grad(const NormGradArgs& a, bool bf16, hipStream_t s) {
  if (a.rows <= 0 || a.cols <= 0) return hipErrorInvalidValue;
  return bf16 ? grad_for<bf16_t>(a, s) : grad_for<float>(a, s);
}

hipError_t launch_col_sums(const float* part, int64_t rows, int64_t cols, void* out, bool bf16, hipStream_t s) {
  if (rows <= 0 || cols <= 0) return hipErrorInvalidValue;
  const dim3 grid((uint32_t)((cols + 31) / 32));
  if (bf16)
    hipLaunchKernelGGL(k_col_sums<bf16_t>, grid, dim3(1024), 0, s, part, rows, cols, (bf16_t*)out);
  else
    hipLaunchKernelGGL(k_col_sums<float>, grid, dim3(1024), 0, s, part, rows, cols, (float*)out);
  return hipGetLastError();
}

}  // namespace ff
