// Matrix-core tile of products whose operands lie along k as they are stored:
// C (M x N) = sum over k of P (k, m) Q (k, n), Q with its rows along n (k from row to
// row: a weight W (m x n) whose m is summed over, the rows x of a gradient), P
// either the same way (g^T x) or with k along its rows (g W).  16-bit floats (gfx950).
//
// As in ff_tile_nt.hpp: four waves, BM x BN = 32 TI x 32 TJ, k in pairs of two steps
// (64 of k), copied global -> LDS without registers, all slots but one in flight.
// An operand by k keeps its rows in LDS, 64 TN bytes of 32 TN columns, and is
// turned as it is read: ds_read_b64_tr_b16 gives lane i of 16 column i of four k
// whose 32 bytes the lanes point at (lane i at four columns 4 (i % 4) of k i / 4).
// Two of them are a lane's eight k of the instruction.  The 32-byte unit u of row r
// sits at u ^ f(r) of its 256 bytes, f(r) = r & 3 | (r >> 3 & 1) << 2 (64-byte rows: half
// of that), so that the eight rows that 32 lanes read at a time cover all 64 banks.
//
// Bound by its matrix instructions and LDS reads (4096 tokens, 4096 x 11008: g W in 277 to 288 us,
// 1.3 PFLOP/s; g^T x in fp16 345 to 360, with the stores of 90 MB), with few k by what
// surrounds them, hence `stream`.
//
// The products are taken transposed, D = Q^T P: a lane holds four consecutive n of
// one m, which it stores at once.
#pragma once

#include "ff_tile_nt.hpp"

namespace ff {
namespace kn {

using nt::kOutside;
using nt::lds_void;
using nt::rsrc;

constexpr int kK = 64;  // k of a pair
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// An operand of a tile from its first row and column on: by rows (k along a row), or by k.
struct Side {
  const char* p;
  int64_t extent;  // rows (by rows) or columns (by k) that exist
  uint32_t ld;     // bytes
};

template <int TN>
__device__ __forceinline__ int turn_swz(int row) {
  return TN == 2 ? (row >> 1 & 1) | (row >> 3 & 1) << 1 : (row & 3) | (row >> 3 & 1) << 2;
}

// (Through a restricted pointer: a read that the compiler knows nothing of waits for every
// copy into LDS that is on its way.  What a read needs has landed and been seen by all
// waves at the pair's barrier.)
__device__ __forceinline__ s16x4 read_turned(lds_s16x4* __restrict__ p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(p);
}

// T: nt::Bf16 or nt::F16.  PK: P by k too.
template <class T, bool PK, int TI, int TJ, int SLOTS>
struct Tile {
  static_assert((TI == 2 || TI == 4 || TI == 8 || !PK) && (TJ == 2 || TJ == 4 || TJ == 8), "whole windows of 256 bytes");
  static constexpr int BM = 32 * TI, BN = 32 * TJ;
  static constexpr int NL = TI + TJ;
  static_assert(SLOTS >= 2 && (SLOTS - 1) * NL < 64, "copies in flight are counted in six bits");
  static constexpr int kWaves = NL * SLOTS <= 20 ? 2 : 1;  // of a SIMD, by LDS
  typedef f32x4 Acc[TI][TJ];

  struct __align__(16) Ring {
    u32x4 p[SLOTS][BM * 8];
    u32x4 q[SLOTS][BN * 8];
  };

  // Where lane `id` of the workgroup copies an operand by k: row of copy 0 (64 / TN further
  // down each), and its column's chunk of 16 bytes.
  template <int TN>
  static __device__ __forceinline__ int k_row(int id) {
    return id / (4 * TN);
  }
  template <int TN>
  static __device__ __forceinline__ int k_chunk(int id, int row) {
    const int c = id % (4 * TN);
    return ((c >> 1) ^ turn_swz<TN>(row)) * 2 + (c & 1);
  }

  struct Lane {
    uint32_t p[TI], q[TJ];
    int pk, qk;  // k within a pair: of the copy (by rows), or of copy 0 (by k)
  };
  static __device__ __forceinline__ Lane lane_of(const Side& P, const Side& Q) {
    Lane L;
    const int id = threadIdx.x;
    if constexpr (PK) {
      L.pk = k_row<TI>(id);
#pragma unroll
      for (int q = 0; q < TI; ++q) {
        const int r = L.pk + q * (kK / TI), c = k_chunk<TI>(id, r);
        L.p[q] = c * 8 < P.extent ? (uint32_t)r * P.ld + 16u * (uint32_t)c : kOutside;
      }
    } else {
      const int r0 = id >> 3, c = (id & 7) ^ nt::swz(r0);
      L.pk = 8 * c;
#pragma unroll
      for (int q = 0; q < TI; ++q)
        L.p[q] = r0 + 32 * q < P.extent ? (uint32_t)(r0 + 32 * q) * P.ld + 16u * (uint32_t)c : kOutside;
    }
    L.qk = k_row<TJ>(id);
#pragma unroll
    for (int q = 0; q < TJ; ++q) {
      const int r = L.qk + q * (kK / TJ), c = k_chunk<TJ>(id, r);
      L.q[q] = c * 8 < Q.extent ? (uint32_t)r * Q.ld + 16u * (uint32_t)c : kOutside;
    }
    return L;
  }

  // Copy q of the pair at pp, pq with `left` of k from there on (P's copies first).
  static __device__ __forceinline__ void issue_one(Ring& sm, int slot, const char* pp, const char* pq, const Lane& L,
                                                   int left, int wave, int q) {
    if (q < TI) {
      const int k = L.pk + (PK ? q * (kK / TI) : 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(pp), (lds_void*)&sm.p[slot][(q * 4 + wave) * 64], 16,
                                               (int)(k < left ? L.p[q] : kOutside), 0, 0, 0);
    } else {
      const int k = L.qk + (q - TI) * (kK / TJ);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(pq), (lds_void*)&sm.q[slot][((q - TI) * 4 + wave) * 64], 16,
                                               (int)(k < left ? L.q[q - TI] : kOutside), 0, 0, 0);
    }
  }

  typedef u32x4 Frags[TI + TJ];

  // Byte offsets of a lane's fragments within a slot of their operand, step 0.
  struct FragBase {
    uint32_t p[PK ? TI : 2], q[TJ];
  };
  template <int TN>
  static __device__ __forceinline__ uint32_t turned_at(int half, int t) {
    const int lane = threadIdx.x & 63, row = 8 * (lane >> 4) + (lane & 15) / 4;
    return (uint32_t)row * (64 * TN) + (uint32_t)((half * TN + t) ^ turn_swz<TN>(row)) * 32 + 8 * (lane & 3);
  }
  static __device__ __forceinline__ FragBase frag_base() {
    FragBase fb;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if constexpr (PK) {
#pragma unroll
      for (int t = 0; t < TI; ++t) fb.p[t] = turned_at<TI>(wave >> 1, t);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        fb.p[h] = (uint32_t)((wave >> 1) * 16 * TI + (lane & 15)) * 128 +
                  16u * (uint32_t)((h * 4 + (lane >> 4)) ^ nt::swz(lane & 15));
    }
#pragma unroll
    for (int t = 0; t < TJ; ++t) fb.q[t] = (uint32_t)sizeof(Ring::p) + turned_at<TJ>(wave & 1, t);
    return fb;
  }

  static __device__ __forceinline__ u32x4 turned(const char* at, int tn) {  // rows of 64 tn bytes
    const s16x4 lo = read_turned((lds_s16x4*)at), hi = read_turned((lds_s16x4*)(at + 4 * 64 * tn));
    typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
    const u32x2 a = __builtin_bit_cast(u32x2, lo), b = __builtin_bit_cast(u32x2, hi);
    return u32x4{a[0], a[1], b[0], b[1]};
  }
  // Fragment x in the order the products use them: P tile 0, the Q tiles, the other P tiles.
  static __device__ __forceinline__ void read_one(const Ring& sm, int slot, int half, const FragBase& fb, Frags& f,
                                                  int x) {
    const int t = x == 0 ? 0 : x <= TJ ? TI + x - 1 : x - TJ;
    const char* base = reinterpret_cast<const char*>(&sm);
    if (t >= TI)
      f[t] = turned(base + fb.q[t - TI] + slot * (BN * 128) + half * (32 * 64 * TJ), TJ);
    else if constexpr (PK)
      f[t] = turned(base + fb.p[t] + slot * (BM * 128) + half * (32 * 64 * TI), TI);
    else
      f[t] = *reinterpret_cast<const u32x4*>(base + fb.p[half] + slot * (BM * 128) + t * (16 * 128));
  }

  template <bool LOADS>
  static __device__ __forceinline__ void step(Ring& sm, const Frags& cur, Frags& nxt, int rslot, int rhalf, int lslot,
                                              const char* pp, const char* pq, const Lane& L, int left, int wave,
                                              const FragBase& fb, Acc& acc) {
    constexpr int NP = TI * TJ;
    constexpr int RS = NP * 3 / 4 / NL > 0 ? NP * 3 / 4 / NL : 1;  // products per read
    constexpr int LS = NP / NL > 0 ? NP / NL : 1;                  // products per copy
    static_assert(NP >= NL, "a read and a copy at most after each product");
#pragma unroll
    for (int m = 0; m < NP; ++m) {
      const int i = m / TJ, j = m % TJ;
      acc[i][j] = T::mfma(cur[TI + j], cur[i], acc[i][j]);
      if (m % RS == 0 && m / RS < NL) read_one(sm, rslot, rhalf, fb, nxt, m / RS);
      if (LOADS && m % LS == 0 && m / LS < NL) issue_one(sm, lslot, pp, pq, L, left, wave, m / LS);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  static __device__ __forceinline__ void pin(Acc& acc) {
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j) {
        if (TI * TJ >= 24)
          asm volatile("" : "+a"(acc[i][j]));
        else
          asm volatile("" : "+v"(acc[i][j]));
      }
  }

  // acc += the products over k of P and Q (both from their first k on), k >= 1.  The
  // loop is nt::Tile's: two steps a pair, the next step's fragments read among the
  // products, one barrier a pair, behind which the slot just read is filled anew.
  static __device__ __forceinline__ void loop(Ring& sm, const Side& P, const Side& Q, int64_t k, Acc& acc) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Lane L = lane_of(P, Q);
    const FragBase fb = frag_base();
    const char *pp = P.p, *pq = Q.p;
    const int64_t step_p = PK ? (int64_t)kK * P.ld : kK * 2, step_q = (int64_t)kK * Q.ld;
    const int count = (int)((k + kK - 1) / kK);
    int64_t left = k;
    auto advance = [&](const char*& a, const char*& b) -> int {  // to the next pair; its k
      a = pp;
      b = pq;
      pp += step_p;
      pq += step_q;
      const int l = (int)max((int64_t)0, min(left, (int64_t)kK));
      left -= kK;
      return l;
    };
    const char *a, *b;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      const int l = advance(a, b);
#pragma unroll
      for (int q = 0; q < NL; ++q) issue_one(sm, s, a, b, L, l, wave, q);
    }
    nt::wait_vmem<(SLOTS - 1) * NL>();
    __builtin_amdgcn_s_barrier();
    Frags F[2];
#pragma unroll
    for (int q = 0; q < NL; ++q) read_one(sm, 0, 0, fb, F[0], q);
    pin(acc);
    int slot = 0;
    for (int p = 0; p < count; ++p) {
      step<false>(sm, F[0], F[1], slot, 1, 0, nullptr, nullptr, L, 0, wave, fb, acc);
      nt::wait_vmem<(SLOTS - 2) * NL>();
      nt::wait_lds();
      __builtin_amdgcn_s_barrier();
      const int l = advance(a, b);
      const int next = slot + 1 == SLOTS ? 0 : slot + 1;
      step<true>(sm, F[1], F[0], next, 0, slot, a, b, L, l, wave, fb, acc);
      slot = next;
    }
    pin(acc);
    nt::wait_vmem<0>();
    __syncthreads();
  }

  // Tile after tile without a pause: the copies run ahead across the ends of tiles, so that
  // the next tile's first pairs land while this one's results are stored.  Tiles: from `work` on,
  // next(P, Q, k) moves to the next tile (k may be 0: all zeros) or returns false.  finish(acc, work)
  // stores a tile; it must leave the ring alone and take no barrier.
  template <class Tiles, class Finish>
  static __device__ __forceinline__ void stream(Ring& sm, Tiles work, Finish finish) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const FragBase fb = frag_base();
    Tiles ahead = work;
    Lane L;
    const char *pp = nullptr, *pq = nullptr, *a = nullptr, *b = nullptr;
    int64_t step_p = 0, step_q = 0, left = 0;
    bool more = true;
    auto advance = [&]() -> int {  // to the next pair of any tile; its k (none left: 0)
      while (left <= 0 && more) {
        Side P, Q;
        more = ahead.next(P, Q, left);
        if (!more || left <= 0) {
          left = 0;
          continue;
        }
        L = lane_of(P, Q);
        pp = P.p;
        pq = Q.p;
        step_p = PK ? (int64_t)kK * P.ld : kK * 2;
        step_q = (int64_t)kK * Q.ld;
      }
      a = pp;
      b = pq;
      pp += step_p;
      pq += step_q;
      const int l = (int)min(left, (int64_t)kK);
      left -= l;
      return l;
    };
#pragma unroll
    for (int q = 0; q < TI; ++q) L.p[q] = kOutside;
#pragma unroll
    for (int q = 0; q < TJ; ++q) L.q[q] = kOutside;
    L.pk = L.qk = 0;
#pragma unroll 1
    for (int s = 0; s < SLOTS; ++s) {
      const int l = advance();
#pragma unroll
      for (int q = 0; q < NL; ++q) issue_one(sm, s, a, b, L, l, wave, q);
    }
    nt::wait_vmem<(SLOTS - 1) * NL>();
    __builtin_amdgcn_s_barrier();
    Frags F[2];
#pragma unroll
    for (int q = 0; q < NL; ++q) read_one(sm, 0, 0, fb, F[0], q);
    int slot = 0;
    Acc acc;
    Side P, Q;
    int64_t k;
    while (work.next(P, Q, k)) {
      zero(acc);
      pin(acc);
      const int count = (int)((k + kK - 1) / kK);
      for (int p = 0; p < count; ++p) {
        step<false>(sm, F[0], F[1], slot, 1, 0, nullptr, nullptr, L, 0, wave, fb, acc);
        // (behind a tile's stores, too, which the first pair after them waits for)
        nt::wait_vmem<(SLOTS - 2) * NL>();
        nt::wait_lds();
        __builtin_amdgcn_s_barrier();
        const int l = advance();
        const int next = slot + 1 == SLOTS ? 0 : slot + 1;
        step<true>(sm, F[1], F[0], next, 0, slot, a, b, L, l, wave, fb, acc);
        slot = next;
      }
      pin(acc);
      finish(acc, work);
    }
    nt::wait_vmem<0>();
  }

  static __device__ __forceinline__ void zero(Acc& acc) {
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
  }
};

}  // namespace kn
}  // namespace ff
