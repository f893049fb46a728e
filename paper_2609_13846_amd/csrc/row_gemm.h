// The bf16 contraction of the dense operators (gfx950): both operands row-major as the caller has
// them, copied into LDS by the buffer unit.
//
// An operand is "along": element (row, k) at [row * ld + k], or "across": at [k * ld + row].
// Whatever its order, a copy instruction moves 64 pieces of 16 bytes, and the lanes choose which
// piece of the source each takes, so that the swizzle of the LDS image costs nothing:
//   along   an LDS row of 64 columns (128 bytes) per operand row, its eight pieces exchanged by the
//           row's number, so that the 16 rows of a fragment lie in different banks;
//   across  an LDS line of all the rows per contraction index, its pairs of pieces exchanged by the
//           line's number, and the fragments read with the transposing LDS read: 16 lanes take
//           4 lines x 16 rows and each gets the 4 lines of its row.  A wavefront's read of B takes
//           each bank twice, the least that its 512 bytes can; one of A takes half of the banks
//           four times, since A's rows are dealt (below) so that it reads the lower or the upper
//           halves of its pieces, which no exchange of whole pieces spreads: 40% of the LDS
//           cycles of dx and dW are conflicts.
// Both read whole 128-byte lines of memory, where stages of 32 columns would read half a line of a row
// at a time.  8,192 x 4,096 x 28,672, both along: 1,384 TFLOP/s (a library product 1,577), the matrix
// cores busy 72% of the time and the wavefronts at a wait for 43%; 65,536 x 1,024 x 6,144, with 16
// stages a tile: 1,160 (1,133 when it ran at 1,414 without its writes).
// Reads past the operand return zeros (the buffer's range for rows and lines behind the last, an
// address out of range for the columns behind a row's last): sizes need not be whole tiles.
//
// Rows of A are dealt to fragments so that a lane holds eight consecutive ones of a result's row:
// fragments 2p and 2p + 1 take rows 8 (r / 4) + r % 4 and + 4 of 32 (r: the row in the fragment).
//
// The loop: eight wavefronts, 2 along A x 4 along B, each AF x BF tiles of 16 x 16; stages of 64
// columns in two LDS slots.  A wavefront's A fragments come in two halves, and a stage is four
// steps of AF / 2 x BF products:
//   1  half 0, columns  0-31   reads half 0, columns 32-63, and B's columns 32-63
//   X  barrier: all have read half 0 and B; half 1 has landed
//   2  half 0, columns 32-63   reads half 1, columns  0-31;  copies half 0 and some of B two stages on
//   3  half 1, columns  0-31   reads half 1, columns 32-63;  copies the rest of B
//   Y  barrier: all have read half 1; the next stage's half 0 and B have landed
//   4  half 1, columns 32-63   reads the next stage's first fragments;  copies half 1 two stages on
// so that every fragment is read a step before its products, a copy has five to seven steps to
// land, and the copies, which a wavefront cannot pass while the path to L2 is busy, are shared out
// over the steps.  In a step the first product goes before the reads and copies of its column (0.6
// to 3% over reads first; one read between any two products took the forward pass 1.4 times as long).  The stages of a block's items follow each other without a gap:
// the copies run two stages ahead into the next item while the results of this one are written.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dense_plan.h"
#include "frag_gemm.h"

namespace dtp {

typedef __attribute__((ext_vector_type(4))) short s16x4;

constexpr uint32_t kRowRange = 0x80000000u;    // most bytes of an operand that a stage may reach
constexpr uint32_t kOutOfRange = 0xc0000000u;  // an offset beyond any range

// Exchange of an across-line's pairs of pieces by the lines 8 g + 0 .. 3 of all g, which one
// transposing read of a wavefront takes: their pairs lie in different banks.
template <int ROWS>
__device__ __forceinline__ int across_swizzle(int line) {
  if constexpr (ROWS == 256) return (line & 3) | ((line >> 3) & 3) << 2;
  if constexpr (ROWS == 128) return (line & 3) | ((line >> 3) & 1) << 2;
  return ((line >> 1) & 1) | ((line >> 3) & 1) << 1;
}
// Exchange of an along-row's pieces: the 16 rows of an A fragment (8 (r / 4) + r % 4), and of a B
// fragment (r), take each of the eight pieces' places twice, once per 128 bytes of the banks.
__device__ __forceinline__ int along_swizzle_a(int row) {
  return (((row >> 1) & 1) | ((row >> 3) & 3) << 1) ^ ((row & 1) << 2);
}
__device__ __forceinline__ int along_swizzle_b(int row) { return ((row >> 1) & 7) ^ ((row & 1) << 2); }

// Where an item's stages are.  `left`: bytes of the operand from the pointer on.
struct RowItem {
  const char *a, *b;  // the item's first row and first stage
  int64_t left_a, left_b;
  int columns;        // left of the segment
  int first, n;       // its first stage's number in the whole contraction, and how many: an even number
};

// The contraction, all in bytes but for the counts: stages of one segment, or of a first and a second
// one that starts jump_a and jump_b behind the end of the first.
struct RowContraction {
  uint32_t lda, ldb;       // elements
  int64_t step_a, step_b;  // from stage to stage
  int64_t half_a;          // from the first half of A's rows to the second (of another matrix: gated)
  int64_t half_left;       // bytes less from there on
  int64_t jump_a, jump_b;
  int columns;             // of a segment
  int per_segment;         // stages, an even number: the last one may have no columns
};

// HALVES: the halves of A's rows are 16 AF consecutive rows each (of two matrices).  Otherwise each
// wavefront's rows are consecutive: half h of its 16 AF rows is 8 AF of them.
template <int AF, int BF, bool AT, bool BT, bool HALVES>
struct RowPipe {
  static constexpr int kARows = 32 * AF, kHalf = kARows / 2, kBRows = 64 * BF;
  static constexpr int kASlot = kHalf * kRowStage, kBSlot = kBRows * kRowStage;  // bf16 per slot
  static constexpr int kACopies = kHalf / 64, kBCopies = kBRows / 64;  // per wavefront: a half's, and B's
  static constexpr int kBFirst = kBCopies > 2 ? 1 : 0;  // of B's, in step 2; the rest in step 3
  static constexpr int kCopies = 2 * kACopies + kBCopies;
  static constexpr int kH = AF / 2;
  static constexpr int kReadsA = AT ? 2 : 1, kReadsB = BT ? 2 : 1;  // LDS reads per fragment
  static_assert(kCopies < 16, "vmcnt field");

  struct Slot {
    uint16_t *a0, *a1, *b;
  };

  int wave, lane, wm, wn;
  const RowContraction& k;
  uint32_t va[kACopies], vb[kBCopies];  // byte offsets of this lane's pieces
  int piece_a, piece_b;                 // (along) first column of the first copy's piece
  int a_at, b_at;                       // a fragment's place in a slot (along)
  int a_line[AT ? kH / 2 : 1], b_line[BT ? BF : 1];  // (across)
  f32x4 acc[AF][BF];
  bf16x8 ax[kH], ay[kH], b0[BF], b1[BF];

  __device__ __forceinline__ static int source_row(int row) {
    return HALVES ? row : row / (8 * AF) * (16 * AF) + row % (8 * AF);
  }

  __device__ __forceinline__ explicit RowPipe(const RowContraction& c) : k(c) {
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    lane = threadIdx.x & 63;
    wm = wave & 1;
    wn = wave >> 1;
    const uint32_t lda = k.lda, ldb = k.ldb;
    piece_a = piece_b = 0;
#pragma unroll
    for (int j = 0; j < kACopies; ++j) {
      const int c0 = wave * kACopies + j;
      if constexpr (AT) {
        const int at = c0 * 512 + lane * 8, line = at / kHalf;
        const int row = 8 * ((at % kHalf / 8) ^ (2 * across_swizzle<kHalf>(line)));
        va[j] = (uint32_t)line * lda * 2u + (uint32_t)source_row(row) * 2u;
      } else {
        const int row = 8 * c0 + lane / 8, p = (lane % 8) ^ along_swizzle_a(row);
        va[j] = (uint32_t)source_row(row) * lda * 2u + (uint32_t)p * 16u;
        if (j == 0) piece_a = 8 * p;
      }
    }
#pragma unroll
    for (int j = 0; j < kBCopies; ++j) {
      const int c0 = wave * kBCopies + j;
      if constexpr (BT) {
        const int at = c0 * 512 + lane * 8, line = at / kBRows;
        const int row = 8 * ((at % kBRows / 8) ^ (2 * across_swizzle<kBRows>(line)));
        vb[j] = (uint32_t)line * ldb * 2u + (uint32_t)row * 2u;
      } else {
        const int row = 8 * c0 + lane / 8, p = (lane % 8) ^ along_swizzle_b(row);
        vb[j] = (uint32_t)row * ldb * 2u + (uint32_t)p * 16u;
        if (j == 0) piece_b = 8 * p;
      }
    }
    const int r = lane % 16, g = lane / 16;
    a_at = b_at = a_line[0] = b_line[0] = 0;
    if constexpr (AT) {
      const int s = 2 * across_swizzle<kHalf>(8 * g + r / 4);
#pragma unroll
      for (int p = 0; p < kH / 2; ++p)
        a_line[p] = (8 * g + r / 4) * kHalf + (((wm * 8 * AF + 32 * p) / 8 + r % 4) ^ s) * 8;
    } else {
      const int row = wm * 8 * AF + 8 * (r / 4) + r % 4;
      a_at = row * kRowStage + (g ^ along_swizzle_a(row)) * 8;
    }
    if constexpr (BT) {
      const int s = 2 * across_swizzle<kBRows>(8 * g + r / 4);
#pragma unroll
      for (int j = 0; j < BF; ++j)
        b_line[j] = (8 * g + r / 4) * kBRows + (((wn * 16 * BF + 16 * j) / 8 + r % 4 / 2) ^ s) * 8 + 4 * (r % 2);
    } else {
      const int row = wn * 16 * BF + r;
      b_at = row * kRowStage + (g ^ along_swizzle_b(row)) * 8;
    }
  }

  // The stage that the copies are at.
  struct Feed {
    RowItem at;  // moved on from stage to stage; n: stages left
    int index;
  };

  // A descriptor of `left` bytes; of none where nothing is left.
  __device__ __forceinline__ static __amdgpu_buffer_rsrc_t stage_rsrc(const char* p, int64_t left) {
    return frag_rsrc(p, left < 0 ? 0u : (left < (int64_t)kRowRange ? (uint32_t)left : kRowRange));
  }
  __device__ __forceinline__ void copy_a(uint16_t* slot, const Feed& f, int half) const {
    const __amdgpu_buffer_rsrc_t rsrc =
        stage_rsrc(f.at.a + (half ? k.half_a : 0), f.at.left_a - (half ? k.half_left : 0));
#pragma unroll
    for (int j = 0; j < kACopies; ++j) {
      const bool out = !AT && (piece_a ^ (16 * j)) >= f.at.columns;  // columns behind the row's last
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rsrc, (__attribute__((address_space(3))) void*)(slot + (kACopies * wave + j) * 512), 16,
          (int)(out ? kOutOfRange : va[j]), 0, 0, 0);
    }
  }
  // The wavefront's copies FROM .. TO - 1 of B.
  template <int FROM, int TO>
  __device__ __forceinline__ void copy_b(uint16_t* slot, const Feed& f) const {
    const __amdgpu_buffer_rsrc_t rsrc = stage_rsrc(f.at.b, f.at.left_b);
#pragma unroll
    for (int j = FROM; j < TO; ++j) {
      const bool out = !BT && (piece_b ^ (32 * (j % 2))) >= f.at.columns;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rsrc, (__attribute__((address_space(3))) void*)(slot + (kBCopies * wave + j) * 512), 16,
          (int)(out ? kOutOfRange : vb[j]), 0, 0, 0);
    }
  }

  // Waits until this wavefront's LDS reads are done and its copies but a stage's, the last, have landed
  // (unless they are known to have), then for the block.
  __device__ __forceinline__ void meet(int& settled) const {
    asm volatile("" ::: "memory");  // no LDS access moves across the barrier
    if (settled > 0) {
      --settled;
      __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    } else {
      __builtin_amdgcn_s_waitcnt(0x0070 | kCopies);  // vmcnt(kCopies), lgkmcnt(0)
    }
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  }

  __device__ __forceinline__ static bf16x8 across_frag(const uint16_t* p, int rows) {
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 4 * rows));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  __device__ __forceinline__ bf16x8 frag_a(const uint16_t* slot, int kk, int i) const {
    if constexpr (AT)
      return across_frag(slot + a_line[i / 2] + kk * 32 * kHalf + 4 * (i % 2), kHalf);
    else
      return *reinterpret_cast<const bf16x8*>(slot + (a_at ^ (32 * kk)) + (32 * (i / 2) + 4 * (i % 2)) * kRowStage);
  }
  __device__ __forceinline__ bf16x8 frag_b(const uint16_t* slot, int kk, int j) const {
    if constexpr (BT)
      return across_frag(slot + b_line[j] + kk * 32 * kBRows, kBRows);
    else
      return *reinterpret_cast<const bf16x8*>(slot + (b_at ^ (32 * kk)) + 16 * j * kRowStage);
  }

  // Keeps a step's order through scheduling: its reads and copies shared out among its products.
  template <int READS, int COPIES>
  __device__ __forceinline__ void order() const {
    constexpr int kReads = (READS + BF - 1) / BF, kSome = (COPIES + BF - 1) / BF;
#pragma unroll
    for (int j = 0; j < BF; ++j) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if constexpr (kSome > 0) __builtin_amdgcn_sched_group_barrier(0x010, kSome, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, kReads, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, kH - 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }

  __device__ __forceinline__ void multiply(int half, const bf16x8 (&a)[kH], const bf16x8 (&bb)[BF]) {
#pragma unroll
    for (int j = 0; j < BF; ++j)
#pragma unroll
      for (int i = 0; i < kH; ++i)
        acc[half * kH + i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], bb[j], acc[half * kH + i][j], 0, 0, 0);
  }
  __device__ __forceinline__ void read_a(const uint16_t* slot, int kk, bf16x8 (&a)[kH]) const {
#pragma unroll
    for (int i = 0; i < kH; ++i) a[i] = frag_a(slot, kk, i);
  }
  __device__ __forceinline__ void read_b(const uint16_t* slot, int kk, bf16x8 (&bb)[BF]) const {
#pragma unroll
    for (int j = 0; j < BF; ++j) bb[j] = frag_b(slot, kk, j);
  }

  // Waits for the copies in flight: before a result is written, so that the next two barriers need not
  // wait for the writes.
  __device__ __forceinline__ static void settle() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
    asm volatile("" ::: "memory");
  }

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < AF; ++i)
#pragma unroll
      for (int j = 0; j < BF; ++j) acc[i][j] = f32x4{};
  }

  // Items index, index + stride, .. below count, one after the other: item(i) says where number i
  // lies, done(i) takes its sums from acc.
  template <typename Item, typename Done>
  __device__ __forceinline__ void run(Slot s0, Slot s1, int index, int count, int stride, Item&& item, Done&& done) {
    Feed f{item(index), index};
    auto move = [&](int64_t a, int64_t b) __attribute__((always_inline)) {
      f.at.a += a;
      f.at.left_a -= a;
      f.at.b += b;
      f.at.left_b -= b;
    };
    auto advance = [&]() __attribute__((always_inline)) {
      if (f.at.n > 1) {
        --f.at.n;
        ++f.at.first;
        f.at.columns -= kRowStage;
        move(k.step_a, k.step_b);
        if (f.at.first == k.per_segment) {  // the second segment: its operands' bytes are counted anew
          f.at.columns = k.columns;
          f.at.a += k.jump_a;
          f.at.left_a += (int64_t)k.per_segment * k.step_a;
          f.at.b += k.jump_b;
          f.at.left_b -= k.jump_b;
        }
      } else if (f.index + stride < count) {
        f.index += stride;
        f.at = item(f.index);
      }  // else nothing follows: the last stage again
    };
    int pairs = f.at.n / 2, settled = 0;
    auto stage = [&](Slot cur, Slot next) __attribute__((always_inline)) {
      read_a(cur.a0, 1, ay);
      read_b(cur.b, 1, b1);
      multiply(0, ax, b0);
      order<kH * kReadsA + BF * kReadsB, 0>();
      meet(settled);  // X
      copy_a(cur.a0, f, 0);
      copy_b<0, kBFirst>(cur.b, f);
      read_a(cur.a1, 0, ax);
      multiply(0, ay, b1);
      order<kH * kReadsA, kACopies + kBFirst>();
      copy_b<kBFirst, kBCopies>(cur.b, f);
      read_a(cur.a1, 1, ay);
      multiply(1, ax, b0);
      order<kH * kReadsA, kBCopies - kBFirst>();
      meet(settled);  // Y
      copy_a(cur.a1, f, 1);
      read_a(next.a0, 0, ax);
      read_b(next.b, 0, b0);
      multiply(1, ay, b1);
      order<kH * kReadsA + BF * kReadsB, kACopies>();
      advance();
    };
    auto whole = [&](Slot s) __attribute__((always_inline)) {
      copy_a(s.a0, f, 0);
      copy_b<0, kBCopies>(s.b, f);
      copy_a(s.a1, f, 1);
      advance();
    };
    whole(s0);
    whole(s1);
    meet(settled);
    read_a(s0.a0, 0, ax);
    read_b(s0.b, 0, b0);
    for (;;) {
      zero();
      for (int i = 0; i < pairs; ++i) {
        stage(s0, s1);
        stage(s1, s0);
      }
      settled = 3;  // done() waits for the copies in flight
      done(index);
      index += stride;
      if (index >= count) break;
      pairs = item(index).n / 2;
      // once more: kept from the last step on, they would take registers from done()
      read_a(s0.a0, 0, ax);
      read_b(s0.b, 0, b0);
    }
    __builtin_amdgcn_s_waitcnt(0x0070);  // nothing lands in LDS after the block is done
    __syncthreads();
  }
};

}  // namespace dtp
