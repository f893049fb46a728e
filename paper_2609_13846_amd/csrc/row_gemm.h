// The bf16 contraction of the dense operators (gfx950): both operands row-major as the caller has
// them, copied into LDS by the buffer unit.
//
// An operand is "along": element (row, k) at [row * ld + k], or "across": at [k * ld + row].
// Whatever its order, a copy instruction moves 64 pieces of 16 bytes, and the lanes choose which
// piece of the source each takes, so that the swizzle of the LDS image costs nothing:
//   along   an LDS row of 32 columns (64 bytes) per operand row, its four pieces exchanged by the
//           row's number, so that the 16 rows of a fragment lie in different banks;
//   across  an LDS line of all the tile's rows per contraction index, its pairs of pieces
//           exchanged by the line's number, and the fragments read with the transposing LDS read:
//           16 lanes take 4 lines x 16 rows and each gets the 4 lines of its row.
// Reads past the operand return zeros (the buffer's range for rows and lines behind the last, an
// address out of range for the columns behind a row's last): sizes need not be whole tiles.
//
// Rows of A are dealt to fragments so that a lane holds eight consecutive ones of a result's row:
// fragments 2p and 2p + 1 take rows 8 r / 4 + r % 4 and + 4 of 32 (r: the row in the fragment).
//
// The loop is that of FragPipe (frag_gemm.h): eight wavefronts, 2 along A x 4 along B, four slots
// of 32 columns, one barrier per stage between the two halves of its products.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "frag_gemm.h"

namespace dtp {

typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;

constexpr uint32_t kRowRange = 0x80000000u;    // most bytes of an operand that a block may reach
constexpr uint32_t kOutOfRange = 0xc0000000u;  // an offset beyond any range

// Exchange of an across-line's pairs of pieces, so that lines 8 g + 0 .. 3 of all g, which one
// transposing read of a wavefront takes, lie in different banks.
template <int ROWS>
__device__ __forceinline__ int across_swizzle(int line) {
  if constexpr (ROWS == 256) return (line & 3) | ((line >> 3) & 3) << 2;
  if constexpr (ROWS == 128) return (line & 3) | ((line >> 3) & 1) << 2;
  return ((line >> 1) & 1) | ((line >> 3) & 1) << 1;
}

struct RowOperand {
  const uint16_t* p;   // the block's first row and column
  const uint16_t* p2;  // of the second segment (or of the second half of A's rows)
  int64_t ld;
  uint32_t range;      // bytes from p on that the block may read
};

// HALVES: A's rows come from two matrices, the first half of the tile's from p, the others from p2.
template <int AF, int BF, bool AT, bool BT, bool HALVES>
struct RowPipe {
  static constexpr int kAFrags = 2 * AF, kBFrags = 4 * BF, kFrags = kAFrags + kBFrags;
  static constexpr int kARows = 16 * kAFrags, kBRows = 16 * kBFrags;
  static constexpr int kSlot = kFrags * 512;  // bf16 per LDS slot
  static constexpr int kCopies = kFrags > 16 ? 4 : 2;  // copies per copying wavefront and stage
  static constexpr int kH0 = AF / 2, kH1 = AF - kH0;
  static constexpr int kReadsA = AT ? 2 : 1, kReadsB = BT ? 2 : 1;  // LDS reads per fragment
  static_assert(kAFrags % kCopies == 0 && kBFrags % kCopies == 0 && kFrags <= 8 * kCopies, "copies share out");
  static_assert(!HALVES || (!AT && (kAFrags / 2) % kCopies == 0 && AF % 4 == 0), "halves share out");

  int wave, lane, wm, wn;
  bool copies_a;
  const uint16_t *src, *src2;
  uint32_t range;
  uint32_t step, jump;      // bytes per stage; of the second segment's first stage
  uint32_t voff[kCopies];
  int piece[2];             // first column of an even and an odd copy's pieces (along)
  int slot_copy;            // first copy's place in a slot, in 512s
  int a_at, b_at;           // a fragment's place in a slot (along)
  int a_line[AT ? AF / 2 : 1], b_line[BT ? BF : 1];  // (across)
  f32x4 acc[AF][BF];
  bf16x8 a0[kH0], a1[kH1], b[BF];

  __device__ __forceinline__ RowPipe(const RowOperand& a, const RowOperand& bm, uint32_t b_jump) {
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    lane = threadIdx.x & 63;
    wm = wave & 1;
    wn = wave >> 1;
    const int w = min(wave, kFrags / kCopies - 1);
    copies_a = w < kAFrags / kCopies;
    const int c0 = kCopies * w - (copies_a ? 0 : kAFrags);  // its first copy in the operand
    slot_copy = kCopies * w;
    const int64_t ld = copies_a ? a.ld : bm.ld;
    src = copies_a ? a.p : bm.p;
    src2 = copies_a ? a.p2 : bm.p;
    range = copies_a ? a.range : bm.range;
    int row0 = 0;
    if (HALVES && copies_a && c0 >= kAFrags / 2) {
      src = a.p2;
      row0 = kARows / 2;
    }
    const bool across = copies_a ? AT : BT;
    step = across ? (uint32_t)ld * 64u : 64u;
    jump = copies_a ? 0u : b_jump;
    piece[0] = piece[1] = 0;
#pragma unroll
    for (int j = 0; j < kCopies; ++j) {
      const int c = c0 + j;
      if (copies_a) {
        if constexpr (AT) {
          voff[j] = across_offset<kARows>(c, ld);
        } else {
          const int row = 16 * c + lane / 4;
          const int s = (2 * ((row >> 1) & 1)) ^ ((row >> 3) & 3);
          voff[j] = (uint32_t)(row - row0) * (uint32_t)ld * 2u + (uint32_t)((lane % 4) ^ s) * 16u;
          if (j < 2) piece[j] = 8 * ((lane % 4) ^ s);
        }
      } else {
        if constexpr (BT) {
          voff[j] = across_offset<kBRows>(c, ld);
        } else {
          const int row = 16 * c + lane / 4;
          const int s = (row >> 1) & 3;
          voff[j] = (uint32_t)row * (uint32_t)ld * 2u + (uint32_t)((lane % 4) ^ s) * 16u;
          if (j < 2) piece[j] = 8 * ((lane % 4) ^ s);
        }
      }
    }
    const int r = lane % 16, g = lane / 16;
    const int rows_a = wm * (HALVES ? 8 * AF : 16 * AF);
    if constexpr (AT) {
      const int s = across_swizzle<kARows>(8 * g + r / 4);
#pragma unroll
      for (int p = 0; p < AF / 2; ++p)
        a_line[p] = (8 * g + r / 4) * kARows + (((rows_a + 32 * p) / 8 + r % 4) ^ (2 * s)) * 8;
      a_at = 0;
    } else {
      a_at = (rows_a + 8 * (r / 4) + r % 4) * 32 + ((g ^ (2 * ((r >> 1) & 1)) ^ (r >> 2)) * 8);
      a_line[0] = 0;
    }
    if constexpr (BT) {
      const int s = across_swizzle<kBRows>(8 * g + r / 4);
#pragma unroll
      for (int j = 0; j < BF; ++j)
        b_line[j] = kARows * 32 + (8 * g + r / 4) * kBRows + (((wn * 16 * BF + 16 * j) / 8 + r % 4 / 2) ^ (2 * s)) * 8 +
                    4 * (r % 2);
      b_at = 0;
    } else {
      b_at = kARows * 32 + (wn * 16 * BF + r) * 32 + ((g ^ ((r >> 1) & 3)) * 8);
      b_line[0] = 0;
    }
  }

  // Byte offset of this lane's piece of copy c of an across operand.
  template <int ROWS>
  __device__ __forceinline__ uint32_t across_offset(int c, int64_t ld) const {
    const int at = c * 512 + lane * 8, line = at / ROWS, p = at % ROWS / 8;
    return (uint32_t)line * (uint32_t)ld * 2u + (uint32_t)(p ^ (2 * across_swizzle<ROWS>(line))) * 16u;
  }

  struct Stage {
    int q;       // stage in its segment
    bool second;
    int columns;  // left of the segment from the stage's first on
  };

  __device__ __forceinline__ void copy(uint16_t* slot, Stage at) const {
    int w = slot_copy;
    asm("" : "+s"(w) : "s"(at.q));
    w = __builtin_amdgcn_readfirstlane(w);
    const uint16_t* base = (!HALVES && at.second) ? src2 : src;
    const __amdgpu_buffer_rsrc_t rsrc = frag_rsrc(base, range);
    const uint32_t off = (uint32_t)at.q * step + (at.second ? jump : 0u);
    const bool along = copies_a ? !AT : !BT;
    // columns behind the row's last are none of this row's
    const bool out0 = along && piece[0] >= at.columns, out1 = along && piece[1] >= at.columns;
#pragma unroll
    for (int j = 0; j < kCopies; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rsrc, (__attribute__((address_space(3))) void*)(slot + (w + j) * 512), 16,
          (int)((AT && BT) ? voff[j] : ((j % 2 ? out1 : out0) ? kOutOfRange : voff[j])),
          __builtin_amdgcn_readfirstlane((int)off), 0, 0);
  }

  template <int STAGES>
  __device__ __forceinline__ void landed() const {
    static_assert(STAGES * kCopies < 16, "vmcnt field");
    asm volatile("" ::: "memory");  // no LDS access moves across the barrier
    __builtin_amdgcn_s_waitcnt(0x0070 | (STAGES * kCopies));  // vmcnt, lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  }

  __device__ __forceinline__ static bf16x8 across_frag(const uint16_t* p, int rows) {
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 4 * rows));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  __device__ __forceinline__ bf16x8 frag_a(const uint16_t* slot, int i) const {
    if constexpr (AT) {
      return across_frag(slot + a_line[i / 2] + 4 * (i % 2), kARows);
    } else {
      const int rows = HALVES ? (i / (AF / 2)) * (kARows / 2) + 32 * (i % (AF / 2) / 2) : 32 * (i / 2);
      return *reinterpret_cast<const bf16x8*>(slot + a_at + (rows + 4 * (i % 2)) * 32);
    }
  }
  __device__ __forceinline__ bf16x8 frag_b(const uint16_t* slot, int j) const {
    if constexpr (BT)
      return across_frag(slot + b_line[j], kBRows);
    else
      return *reinterpret_cast<const bf16x8*>(slot + b_at + 16 * j * 32);
  }

  template <int FIRST, int ROWS, int LATER, int COPIES>
  __device__ __forceinline__ void order() const {
    __builtin_amdgcn_sched_group_barrier(0x100, FIRST, 0);
#pragma unroll
    for (int j = 0; j < BF; ++j) {
      __builtin_amdgcn_sched_group_barrier(0x008, ROWS, 0);
      if (j < COPIES) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
      if constexpr (LATER > 0) __builtin_amdgcn_sched_group_barrier(0x100, LATER, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }

  __device__ __forceinline__ void read_half0(const uint16_t* slot) {
#pragma unroll
    for (int i = 0; i < kH0; ++i) a0[i] = frag_a(slot, i);
  }

  __device__ __forceinline__ void half0(const uint16_t* cur) {
#pragma unroll
    for (int i = 0; i < kH1; ++i) a1[i] = frag_a(cur, kH0 + i);
#pragma unroll
    for (int j = 0; j < BF; ++j)
#pragma unroll
      for (int i = 0; i < kH0; ++i)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0[i], b[j], acc[i][j], 0, 0, 0);
    order<kH1 * kReadsA, kH0, 0, 0>();
  }

  __device__ __forceinline__ void half1(uint16_t* cur, const uint16_t* next, Stage at) {
    landed<2>();
    copy(cur, at);
    read_half0(next);
#pragma unroll
    for (int j = 0; j < BF; ++j) {
#pragma unroll
      for (int i = 0; i < kH1; ++i)
        acc[kH0 + i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1[i], b[j], acc[kH0 + i][j], 0, 0, 0);
      b[j] = frag_b(next, j);
    }
    order<kH0 * kReadsA, kH1, kReadsB, kCopies>();
  }

  // Stages q0 .. q1 of a contraction of nq_seg stages (`columns` columns) per segment; q_base: the
  // stage at which the operands' pointers stand (0 where there are two segments).
  __device__ __forceinline__ void contract(uint16_t* s0, uint16_t* s1, uint16_t* s2, uint16_t* s3, int q0, int q1,
                                           int nq_seg, int64_t columns, int q_base) {
    auto at = [&](int q) __attribute__((always_inline)) {
      q = min(q, q1 - 1);
      const bool second = q >= nq_seg;
      const int in_seg = second ? q - nq_seg : q;
      const int64_t left = columns - 32 * (int64_t)in_seg;
      return Stage{in_seg - q_base, second, left < 32 ? (int)left : 32};
    };
    auto stage = [&](uint16_t* cur, uint16_t* next, int q) __attribute__((always_inline)) {
      const Stage later = at(q + 4);
      half0(cur);
      half1(cur, next, later);
    };
#pragma unroll
    for (int i = 0; i < AF; ++i)
#pragma unroll
      for (int j = 0; j < BF; ++j) acc[i][j] = f32x4{};
    copy(s0, at(q0));
    copy(s1, at(q0 + 1));
    copy(s2, at(q0 + 2));
    copy(s3, at(q0 + 3));
    landed<3>();
    read_half0(s0);
#pragma unroll
    for (int j = 0; j < BF; ++j) b[j] = frag_b(s0, j);
    int q = q0;
    for (; q + 3 < q1; q += 4) {
      stage(s0, s1, q);
      stage(s1, s2, q + 1);
      stage(s2, s3, q + 2);
      stage(s3, s0, q + 3);
    }
    if (q < q1) stage(s0, s1, q);
    if (q + 1 < q1) stage(s1, s2, q + 1);
    if (q + 2 < q1) stage(s2, s3, q + 2);
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): nothing lands in LDS after the block is done
    __syncthreads();
  }
};

}  // namespace dtp
