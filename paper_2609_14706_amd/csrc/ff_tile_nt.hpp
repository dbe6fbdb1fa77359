// Matrix-core tile of the layer operators' products: C = A B^T with both
// operands contiguous along k, 16-bit floats or 8-bit integers (gfx950).
//
// One workgroup of four waves computes a BM x BN tile, BM = 32 TI and
// BN = 32 TJ, each wave TI x TJ tiles of 16 x 16.  Every type's instruction
// takes 16 bytes of k from each lane (v_mfma_f32_16x16x32_{bf16,f16},
// v_mfma_i32_16x16x64_i8), so k is counted in bytes here and one loop serves
// all: k goes in pairs of 64-byte steps, i.e. whole 128-byte lines of each
// operand row, copied global -> LDS without registers (buffer_load ... lds,
// 16 bytes a lane) through two slots, one pair in flight ahead of the matrix
// cores.  The 16-byte chunk c of row r sits at position c ^ ((r >> 1) & 7) of
// its row: a fragment read (one chunk of 16 consecutive rows per pass) then
// covers all 64 banks.
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

// One operand of a tile: its first row, the rows from there on that exist and
// the bytes from row to row.
struct Rows {
  const char* p;
  int rows;
  uint32_t ld;
};

template <class T, int TI, int TJ>
struct Tile {
  static constexpr int BM = 32 * TI, BN = 32 * TJ;
  typedef typename T::acc Acc[TI][TJ];

  struct __align__(16) Ring {
    u32x4 a[2][BM * kChunks];
    u32x4 b[2][BN * kChunks];
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

  // The products of one step.  If READ, the fragments of the next step are
  // read among the first three quarters of them; if LOADS, the copies of a
  // later pair are spread over all of them.
  template <bool READ, bool LOADS>
  static __device__ __forceinline__ void step(Ring& sm, const Frags& cur, Frags& nxt, int rslot, int rhalf,
                                              int lslot, const char* pa, const char* pb, const Lane& L,
                                              uint32_t cut, int wave, const FragBase& fb, Acc& acc) {
    constexpr int NP = TI * TJ, NR = TI + TJ;
    constexpr int RS = NP * 3 / 4 / NR > 0 ? NP * 3 / 4 / NR : 1;   // products per read
    constexpr int RB = (NR + NP - 1) / NP;                          // reads per product (tiny tiles)
    constexpr int LS = NP / NR > 0 ? NP / NR : 1;
#pragma unroll
    for (int m = 0; m < NP; ++m) {
      const int i = m / TJ, j = m % TJ;
      acc[i][j] = T::mfma(cur[i], cur[TI + j], acc[i][j]);
      if (READ) {
        if (RB > 1) {
#pragma unroll
          for (int q = m * RB; q < (m + 1) * RB && q < NR; ++q) read_one(sm, rslot, rhalf, fb, nxt, q);
        } else if (m % RS == 0 && m / RS < NR) {
          read_one(sm, rslot, rhalf, fb, nxt, m / RS);
        }
      }
      if (LOADS) {
        if (RB > 1) {
#pragma unroll
          for (int q = m * RB; q < (m + 1) * RB && q < NR; ++q) issue_one(sm, lslot, pa, pb, L, cut, wave, q);
        } else if (m % LS == 0 && m / LS < NR) {
          issue_one(sm, lslot, pa, pb, L, cut, wave, m / LS);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // acc += sum over pairs [p0, p1).  addr(p, pa, pb) yields the operands'
  // pointers at pair p (row 0); left(p) the bytes of k that are left there
  // (128 or more for a whole pair).  Per pair, its first step multiplies from
  // registers while the second step's fragments are read; then the next pair
  // has to have landed, the pair's one barrier is taken (every wave has read
  // all of this slot and sees the next pair), and the second step reads the
  // next pair's first fragments and copies the pair after it into the slot
  // just freed.  Every wave takes the same number of barriers: n is uniform.
  template <class Addr, class Left>
  static __device__ __forceinline__ void loop(Ring& sm, const Rows& A, const Rows& B, int p0, int p1,
                                              const Addr& addr, const Left& left, Acc& acc) {
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = p1 - p0;
    if (n <= 0) return;
    const Lane L = lane_of(A, B, wave, lane);
    const FragBase fb = frag_base(wave, lane);
    const char *pa, *pb;
    auto cut = [&](int p) -> uint32_t { return 16 * L.c < left(p) ? 0u : kOutside; };
    auto pair = [&](int p, int slot) {
      addr(p, pa, pb);
      const uint32_t c = cut(p);
#pragma unroll
      for (int q = 0; q < TI + TJ; ++q) issue_one(sm, slot, pa, pb, L, c, wave, q);
    };
    pair(p0, 0);
    if (n > 1) {
      pair(p0 + 1, 1);
      wait_vmem<TI + TJ>();
    } else {
      wait_vmem<0>();
    }
    __builtin_amdgcn_s_barrier();
    Frags F[2];
#pragma unroll
    for (int q = 0; q < TI + TJ; ++q) read_one(sm, 0, 0, fb, F[0], q);
    int j = 0;
    for (; j + 2 < n; ++j) {
      const int slot = j & 1;
      step<true, false>(sm, F[0], F[1], slot, 1, 0, nullptr, nullptr, L, 0, wave, fb, acc);
      wait_vmem<0>();
      wait_lds();
      __builtin_amdgcn_s_barrier();
      addr(p0 + j + 2, pa, pb);
      step<true, true>(sm, F[1], F[0], slot ^ 1, 0, slot, pa, pb, L, cut(p0 + j + 2), wave, fb, acc);
    }
    if (j + 1 < n) {
      const int slot = j & 1;
      step<true, false>(sm, F[0], F[1], slot, 1, 0, nullptr, nullptr, L, 0, wave, fb, acc);
      wait_vmem<0>();
      wait_lds();
      __builtin_amdgcn_s_barrier();
      step<true, false>(sm, F[1], F[0], slot ^ 1, 0, 0, nullptr, nullptr, L, 0, wave, fb, acc);
      ++j;
    }
    step<true, false>(sm, F[0], F[1], j & 1, 1, 0, nullptr, nullptr, L, 0, wave, fb, acc);
    step<false, false>(sm, F[1], F[0], 0, 0, 0, nullptr, nullptr, L, 0, wave, fb, acc);
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
