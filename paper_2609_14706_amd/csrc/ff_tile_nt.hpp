// Matrix-core tile of the layer operators' products: C = A B^T with both
// operands contiguous along k, 16-bit floats or 8-bit integers (gfx950).
//
// One workgroup of four waves computes a BM x BN tile, BM = 32 TI and
// BN = 32 TJ, each wave TI x TJ tiles of 16 x 16.  Every type's instruction
// takes 16 bytes of k from each lane (v_mfma_f32_16x16x32_{bf16,f16},
// v_mfma_i32_16x16x64_i8), so k is counted in bytes here and one loop serves
// all: k goes in pairs of 64-byte steps, i.e. whole 128-byte lines of each
// operand row, copied global -> LDS without registers (buffer_load ... lds,
// 16 bytes a lane) through SLOTS slots, all but one of them in flight ahead of the
// matrix cores: two where the products of a pair take longer than its copies,
// more where a tile is small or there are few of them.  The 16-byte chunk c of
// row r sits at position c ^ ((r >> 1) & 7) of its row: a fragment read (one
// chunk of 16 consecutive rows per pass) then covers all 64 banks.
//
// Rows beyond the operand and k beyond its end are zeros: their lanes copy
// from an offset that the buffer descriptor's range check rejects, which
// returns zero and touches no memory.  Rows have to start 16-byte aligned and
// k has to be whole 16-byte chunks.
#pragma once

#include "ff_vec.hpp"

namespace ff {
namespace nt {

typedef __attribute__((ext_vector_type(4))) int32_t i32x4;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((address_space(3))) void lds_void;

// Element types: accumulator of one lane and the instruction.
struct Bf16 {
  typedef f32x4 acc;
  static constexpr int kBytes = 2;
  static __device__ __forceinline__ acc mfma(u32x4 a, u32x4 b, acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
struct F16 {
  typedef f32x4 acc;
  static constexpr int kBytes = 2;
  static __device__ __forceinline__ acc mfma(u32x4 a, u32x4 b, acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
struct I8 {
  typedef i32x4 acc;
  static constexpr int kBytes = 1;
  static __device__ __forceinline__ acc mfma(u32x4 a, u32x4 b, acc c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a),
                                                 __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
  }
};

constexpr int kThreads = 256;       // four waves, 2 x 2
constexpr int kPair = 128;          // bytes of k copied at a time
constexpr int kChunks = kPair / 16; // 16-byte chunks of a pair
constexpr uint32_t kOutside = 0x80000000u;  // beyond every buffer's range
constexpr int64_t kMaxRowBytes = int64_t(1) << 22;  // 256 rows stay below 2^31 bytes

template <int N>
__device__ __forceinline__ void wait_vmem() {  // vmcnt(N), the other counters left alone
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}
__device__ __forceinline__ void wait_lds() {  // lgkmcnt(0) likewise
  __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));
}

__device__ __forceinline__ int swz(int row) { return (row >> 1) & 7; }

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const char* p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), (short)0, (int)0x7fffffff, 0x00020000);
}

// k without interruption, from pair 0 at pa and pb on.
struct Straight {
  const char* pa;
  const char* pb;
  int left;
  __device__ __forceinline__ int operator()(const char*& a, const char*& b) {
    a = pa;
    b = pb;
    pa += kPair;
    pb += kPair;
    const int l = left;
    left -= kPair;
    return l;
  }
};

// One operand of a tile: its first row, the rows from there on that exist and
// the bytes from row to row.
struct Rows {
  const char* p;
  int rows;
  uint32_t ld;
};

template <class T, int TI, int TJ, int SLOTS>
struct Tile {
  static constexpr int BM = 32 * TI, BN = 32 * TJ;
  static constexpr int NL = TI + TJ;  // copies a wave issues per pair
  static_assert(SLOTS >= 2 && (SLOTS - 1) * NL < 64, "copies in flight are counted in six bits");
  typedef typename T::acc Acc[TI][TJ];

  struct __align__(16) Ring {
    u32x4 a[SLOTS][BM * kChunks];
    u32x4 b[SLOTS][BN * kChunks];
  };

  // B's rows are permuted within each wave's half so that a lane's TJ tiles
  // are TJ consecutive columns of C: LDS row 16 j + c holds row TJ c + j.
  static __device__ __forceinline__ int b_row(int r) {
    const int h = r / (16 * TJ), q = r % (16 * TJ);
    return h * 16 * TJ + TJ * (q & 15) + (q >> 4);
  }

  // What a lane copies: chunk `c` of TI + TJ rows, one per instruction.
  struct Lane {
    uint32_t a[TI], b[TJ];
    int c;
  };
  static __device__ __forceinline__ Lane lane_of(const Rows& A, const Rows& B, int wave, int lane) {
    Lane L;
    const int r0 = wave * 8 + (lane >> 3);  // LDS row of instruction 0; 32 further down each
    L.c = (lane & 7) ^ swz(r0);
#pragma unroll
    for (int q = 0; q < TI; ++q) {
      const int r = r0 + 32 * q;
      L.a[q] = r < A.rows ? (uint32_t)r * A.ld + 16u * (uint32_t)L.c : kOutside;
    }
#pragma unroll
    for (int q = 0; q < TJ; ++q) {
      const int r = b_row(r0 + 32 * q);
      L.b[q] = r < B.rows ? (uint32_t)r * B.ld + 16u * (uint32_t)L.c : kOutside;
    }
    return L;
  }

  // Copy q of a pair (B's rows after A's).  cut: kOutside in lanes whose
  // chunk lies beyond the end of k, else 0.
  static __device__ __forceinline__ void issue_one(Ring& sm, int slot, const char* pa, const char* pb,
                                                   const Lane& L, uint32_t cut, int wave, int q) {
    if (q < TI)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(pa), (lds_void*)&sm.a[slot][(q * 4 + wave) * 64], 16,
                                               (int)(L.a[q] | cut), 0, 0, 0);
    else
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(pb), (lds_void*)&sm.b[slot][((q - TI) * 4 + wave) * 64],
                                               16, (int)(L.b[q - TI] | cut), 0, 0, 0);
  }

  typedef u32x4 Frags[TI + TJ];

  // Byte offset of a lane's chunk of tile 0, [operand][step of the pair].
  struct FragBase {
    uint32_t v[2][2];
  };
  static __device__ __forceinline__ FragBase frag_base(int wave, int lane) {
    FragBase fb;
    const uint32_t s = (uint32_t)swz(lane & 15), kc = (uint32_t)(lane >> 4);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t c = 16u * (((uint32_t)h * 4 + kc) ^ s);
      fb.v[0][h] = (uint32_t)((wave >> 1) * 16 * TI + (lane & 15)) * kPair + c;
      fb.v[1][h] = (uint32_t)sizeof(Ring::a) + (uint32_t)((wave & 1) * 16 * TJ + (lane & 15)) * kPair + c;
    }
    return fb;
  }
  // Fragment q in the order the products use them: A tile 0, the B tiles, the
  // other A tiles.
  static __device__ __forceinline__ void read_one(const Ring& sm, int slot, int half, const FragBase& fb,
                                                  Frags& f, int q) {
    const int t = q == 0 ? 0 : q <= TJ ? TI + q - 1 : q - TJ;
    const uint32_t off = t < TI
                             ? fb.v[0][half] + (uint32_t)slot * (BM * kPair) + (uint32_t)t * (16 * kPair)
                             : fb.v[1][half] + (uint32_t)slot * (BN * kPair) + (uint32_t)(t - TI) * (16 * kPair);
    f[t] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(&sm) + off);
  }

  // The products of one step, with the next step's fragments read among the
  // first three quarters of them.  If LOADS, the copies of a later pair are
  // spread over all of them.
  template <bool LOADS>
  static __device__ __forceinline__ void step(Ring& sm, const Frags& cur, Frags& nxt, int rslot, int rhalf,
                                              int lslot, const char* pa, const char* pb, const Lane& L,
                                              uint32_t cut, int wave, const FragBase& fb, Acc& acc) {
    constexpr int NP = TI * TJ;
    constexpr int RS = NP * 3 / 4 / NL > 0 ? NP * 3 / 4 / NL : 1;  // products per read
    constexpr int LS = NP / NL > 0 ? NP / NL : 1;                  // products per copy
    static_assert(NP >= NL, "a read and a copy at most after each product");
#pragma unroll
    for (int m = 0; m < NP; ++m) {
      const int i = m / TJ, j = m % TJ;
      acc[i][j] = T::mfma(cur[i], cur[TI + j], acc[i][j]);
      if (m % RS == 0 && m / RS < NL) read_one(sm, rslot, rhalf, fb, nxt, m / RS);
      if (LOADS && m % LS == 0 && m / LS < NL) issue_one(sm, lslot, pa, pb, L, cut, wave, m / LS);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // Said before and after the loop, this keeps the accumulators in one file
  // through it: of a large tile in the accumulation file, of others not.  Without
  // it the compiler moved 100 to 300 of them between the files at every pair.
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

  // acc += sum over `count` pairs.  walk(pa, pb) yields the operands' pointers
  // (row 0) at the next pair, in order, and returns the bytes of k that are left
  // there (128 or more for a whole pair).  Per pair, its first step multiplies from
  // registers while the second step's fragments are read; then the next pair
  // has to have landed (copies return in order: at most SLOTS - 2 later pairs
  // are still on their way), the pair's one barrier is taken (every wave has
  // read all of this slot and sees the next pair), and the second step reads
  // the next pair's first fragments and copies the pair SLOTS further on into
  // the slot just freed.  Pairs beyond the last are "copied" from outside, i.e.
  // their slots get zeros that no product uses: one loop body for all pairs keeps
  // the accumulators where they are (peeled ends moved hundreds of registers).
  // Every wave takes the same number of barriers: count is uniform.
  //
  // Small tiles (up to eight products a step) would wait for the fragments' LDS
  // latency at every step: they take whole pairs, the next pair's fragments
  // read among this one's products, two pairs a turn so that no fragment changes
  // registers, and the last pair waits for nothing (updates of 70 x 200 fp32: 119
  // us, 130 by steps).  Tiles of 4 x 4 have products enough to hide it: whole
  // pairs left them as they were or cost 6 % (2048 x 3000 fp32: 984 and 1046 us).
  template <class Walk>
  static __device__ __forceinline__ void loop(Ring& sm, const Rows& A, const Rows& B, int count, Walk& walk,
                                              Acc& acc) {
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (count <= 0) return;
    const Lane L = lane_of(A, B, wave, lane);
    const FragBase fb = frag_base(wave, lane);
    const char *pa, *pb;
    const int chunk = 16 * L.c;
    auto advance = [&](int p) -> uint32_t {  // to pair p, the next one
      const int left = walk(pa, pb);
      return chunk < (p < count ? left : 0) ? 0u : kOutside;
    };
#pragma unroll
    for (int q = 0; q < SLOTS; ++q) {
      const uint32_t c = advance(q);
#pragma unroll
      for (int k = 0; k < NL; ++k) issue_one(sm, q, pa, pb, L, c, wave, k);
    }
    wait_vmem<(SLOTS - 1) * NL>();
    __builtin_amdgcn_s_barrier();
    int slot = 0;
    if constexpr (TI * TJ <= 8) {
      Frags F[2][2];
#pragma unroll
      for (int q = 0; q < 2 * NL; ++q) read_one(sm, 0, q / NL, fb, F[0][q / NL], q % NL);
      pin(acc);
      auto whole = [&](const Frags(&cur)[2], Frags(&nxt)[2], int p) {
        wait_vmem<(SLOTS - 2) * NL>();
        wait_lds();
        __builtin_amdgcn_s_barrier();
        const uint32_t c = advance(p + SLOTS);
        const int next = slot + 1 == SLOTS ? 0 : slot + 1;
        constexpr int NP = TI * TJ;
        static_assert(2 * NP >= 2 * NL, "reads and copies after products");
#pragma unroll
        for (int m = 0; m < 2 * NP; ++m) {
          const int h = m / NP, i = m % NP / TJ, j = m % TJ;
          acc[i][j] = T::mfma(cur[h][i], cur[h][TI + j], acc[i][j]);
          if (m < NL) {
            read_one(sm, next, 0, fb, nxt[0], m);
            read_one(sm, next, 1, fb, nxt[1], m);
          } else if (m < 2 * NL) {
            issue_one(sm, slot, pa, pb, L, c, wave, m - NL);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        slot = next;
      };
      auto last = [&](const Frags(&cur)[2]) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < TI; ++i)
#pragma unroll
            for (int j = 0; j < TJ; ++j) acc[i][j] = T::mfma(cur[h][i], cur[h][TI + j], acc[i][j]);
      };
      int p = 0;
      for (; p + 2 < count; p += 2) {
        whole(F[0], F[1], p);
        whole(F[1], F[0], p + 1);
      }
      wait_lds();
      if (p + 2 == count) {
        whole(F[0], F[1], p);
        wait_lds();
        last(F[1]);
      } else {
        last(F[0]);
      }
      pin(acc);
      wait_vmem<0>();
      __syncthreads();
      return;
    }
    Frags F[2];
#pragma unroll
    for (int q = 0; q < NL; ++q) read_one(sm, 0, 0, fb, F[0], q);
    pin(acc);
    for (int p = 0; p < count; ++p) {
      step<false>(sm, F[0], F[1], slot, 1, 0, nullptr, nullptr, L, 0, wave, fb, acc);
      wait_vmem<(SLOTS - 2) * NL>();
      wait_lds();
      __builtin_amdgcn_s_barrier();
      const uint32_t c = advance(p + SLOTS);
      const int next = slot + 1 == SLOTS ? 0 : slot + 1;
      step<true>(sm, F[1], F[0], next, 0, slot, pa, pb, L, c, wave, fb, acc);
      slot = next;
    }
    pin(acc);
    wait_vmem<0>();  // the copies of zeros: LDS is the caller's from here on
    __syncthreads();
  }

  static __device__ __forceinline__ void zero(Acc& acc) {
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j) acc[i][j] = typename T::acc{0, 0, 0, 0};
  }

  // Row of element r of A tile i, and first of the TJ consecutive columns
  // (tile j holds column first + j), within the workgroup's tile.
  static __device__ __forceinline__ int row_of(int i, int r) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    return (wave >> 1) * 16 * TI + i * 16 + 4 * (lane >> 4) + r;
  }
  static __device__ __forceinline__ int col_of() {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    return (wave & 1) * 16 * TJ + TJ * (lane & 15);
  }
};

}  // namespace nt
}  // namespace ff
