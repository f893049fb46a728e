// The fp32 products of the dense operators, on the fp32 matrix instructions: tiles of 128 x 128 (64 x
// 64 where those would leave CUs idle), each wavefront a quarter of a tile in 32 x 32 pieces.
//
// An operand that lies along the contraction is kept [row][k] in LDS, so that a lane's 16-byte read
// is the operand of four instructions; one that lies across it stays [k][row], a dword per
// instruction.  Lane l feeds row l % 32 and, in step j of eight columns, column 4 (l / 32) + j, of
// both operands alike.  The matrix cores need 64 cycles per instruction and 2 to 8 LDS reads
// per eight instructions, so that loads through registers, one stage ahead, keep up: 8,192 x 4,096
// x 4,096 in 2.08 to 2.12 ms, 130 TFLOP/s, in either order (a library product 1.82); 2,048 x 1,536 x
// 512 in 41 us, 256 blocks of 48 stages (29).
#include <algorithm>

#include "dense_stream.h"

namespace dtp {
namespace {

constexpr int kStage = kStageF32;      // columns per stage
constexpr int kAlongRow = kStage + 4;  // floats: 16 rows' 16-byte reads cover the banks once

typedef __attribute__((ext_vector_type(16))) float f32x16;

struct TileArgs {
  const float *a0, *a1, *b;
  int64_t lda, ldb, K, b_seg;
  int M, Mp, segments;
  int64_t N;
  int m_tiles, per, stages;  // stages per split, and of a segment
  uint32_t first;            // tile of the launch
  float* partial;
  ProductOut out;
};

// One operand's stage on its way from memory to LDS: ROWS x kStage elements by THREADS threads.
template <int ROWS, bool ACROSS, int THREADS>
struct Stage {
  static constexpr int kPieces = ROWS * kStage / 4 / THREADS;
  static constexpr int kAcrossRow = ROWS + 8;  // floats: lines 4 apart lie in the other half of the banks
  static constexpr int kFloats = ACROSS ? kStage * kAcrossRow : ROWS * kAlongRow;
  static constexpr int kAlong = kStage / 4;  // pieces of a row
  f32x4 v[kPieces];

  // Rows row0 .. of an operand of `rows` x K, columns k0 .. of the stage.  Whole stages take their
  // addresses as a uniform base and a lane's offset (`lane_at`, fixed for the launch): formed anew per
  // piece, with its bounds, they took the vector unit longer than the products the matrix cores.
  __device__ __forceinline__ static uint32_t lane_at(int64_t ld) {
    const uint32_t at = threadIdx.x;
    return ACROSS ? at / (ROWS / 4) * (uint32_t)ld + at % (ROWS / 4) * 4 : at / kAlong * (uint32_t)ld + at % kAlong * 4;
  }
  __device__ __forceinline__ void load(const float* p, int64_t ld, int64_t row0, int64_t rows, int64_t k0, int64_t K,
                                       uint32_t lane) {
    if (row0 + ROWS <= rows && k0 + kStage <= K) {
      const float* base = p + (ACROSS ? k0 * ld + row0 : row0 * ld + k0);
      const int64_t next = ACROSS ? THREADS / (ROWS / 4) * ld : THREADS / kAlong * ld;
#pragma unroll
      for (int i = 0; i < kPieces; ++i) v[i] = *reinterpret_cast<const f32x4_any*>(base + i * next + lane);
      return;
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int at = threadIdx.x + THREADS * i;
      const int64_t row = row0 + (ACROSS ? at % (ROWS / 4) * 4 : at / kAlong), k = k0 + (ACROSS ? at / (ROWS / 4) : at % kAlong * 4);
      const int64_t along = ACROSS ? row : k, end = ACROSS ? rows : K;
      const bool line = ACROSS ? k < K : row < rows;
      const float* q = p + (ACROSS ? k * ld + row : row * ld + k);
      v[i] = f32x4{};
      if (line && along + 3 < end) {
        v[i] = *reinterpret_cast<const f32x4_any*>(q);
      } else if (line) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (along + e < end) v[i][e] = q[e];
      }
    }
  }
  __device__ __forceinline__ void store(float* lds) const {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int at = threadIdx.x + THREADS * i;
      float* q = ACROSS ? lds + at / (ROWS / 4) * kAcrossRow + at % (ROWS / 4) * 4 : lds + at / kAlong * kAlongRow + at % kAlong * 4;
      *reinterpret_cast<f32x4*>(q) = v[i];
    }
  }
  // Columns 8 s + 4 (lane / 32) .. + 3 of row `row` + lane % 32.
  __device__ __forceinline__ static f32x4 read(const float* lds, int row, int s, int lane) {
    const int r = row + lane % 32, k = 8 * s + 4 * (lane / 32);
    if constexpr (!ACROSS) return *reinterpret_cast<const f32x4*>(lds + r * kAlongRow + k);
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = lds[(k + e) * kAcrossRow + r];
    return v;
  }
};

// F x F pieces of 32 x 32 per wavefront (gated: of each projection, F / 2 x F).  With F = 1, where a
// launch has few tiles, eight wavefronts: two sets that share a stage's columns, whose sums meet
// in LDS, so that a SIMD has one to multiply while the other reads.
template <int F, bool AT, bool BT, ProductKind KIND>
__global__ void __launch_bounds__(F > 1 ? 256 : 512, 2) tile_product_f32_kernel(TileArgs p) {
  constexpr int kSets = F > 1 ? 1 : 2, kThreads = 256 * kSets;
  constexpr bool kGated = KIND == kProductGated;
  constexpr int kTile = 64 * F, kMats = kGated ? 2 : 1, kFM = kGated ? (F > 1 ? F / 2 : 1) : F;
  constexpr int kRowsA = 64 * kFM;  // of each matrix
  using SA = Stage<kRowsA, AT, kThreads>;
  using SB = Stage<kTile, BT, kThreads>;
  __shared__ __attribute__((aligned(16))) float lds[2][kMats * SA::kFloats + SB::kFloats];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wm = wave & 1, wn = wave >> 1 & 1, set = wave >> 2;
  const uint32_t tile = p.first + blockIdx.x;
  const int64_t m0 = (int64_t)(tile % p.m_tiles) * kRowsA, n0 = (int64_t)(tile / p.m_tiles) * kTile;
  const int q0 = blockIdx.y * p.per, q1 = min(q0 + p.per, p.stages * p.segments);
  f32x16 acc[kMats][kFM][F] = {};
  struct {  // the stage on its way
    SA a[kMats];
    SB b;
  } x;
  const uint32_t lane_a = SA::lane_at(p.lda), lane_b = SB::lane_at(p.ldb);
  auto load = [&](int q) __attribute__((always_inline)) {
    const int seg = q >= p.stages ? 1 : 0;
    const int64_t k0 = (int64_t)(q - seg * p.stages) * kStage;
#pragma unroll
    for (int i = 0; i < kMats; ++i)
      x.a[i].load((kGated ? i : seg) ? p.a1 : p.a0, p.lda, m0, p.M, k0, p.K, lane_a);
    x.b.load(p.b + (BT ? 0 : seg * p.b_seg), p.ldb, n0, p.N, k0, p.K, lane_b);
  };
  auto store = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kMats; ++i) x.a[i].store(lds[buf] + i * SA::kFloats);
    x.b.store(lds[buf] + kMats * SA::kFloats);
  };
  load(q0);
  store(0);
  __syncthreads();
  auto stage = [&](int q, int buf) __attribute__((always_inline)) {  // from LDS buffer `buf`
    if (q + 1 < q1) load(q + 1);
#pragma unroll
    for (int i8 = 0; i8 < kStage / 8 / kSets; ++i8) {
      const int s = set * (kStage / 8 / kSets) + i8;
      f32x4 a[kMats][kFM], b[F];
#pragma unroll
      for (int m = 0; m < kMats; ++m)
#pragma unroll
        for (int i = 0; i < kFM; ++i) a[m][i] = SA::read(lds[buf] + m * SA::kFloats, 32 * (wm * kFM + i), s, lane);
#pragma unroll
      for (int j = 0; j < F; ++j) b[j] = SB::read(lds[buf] + kMats * SA::kFloats, 32 * (wn * F + j), s, lane);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int m = 0; m < kMats; ++m)
#pragma unroll
          for (int i = 0; i < kFM; ++i)
#pragma unroll
            for (int j = 0; j < F; ++j)
              acc[m][i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[m][i][e], b[j][e], acc[m][i][j], 0, 0, 0);
    }
    if (q + 1 < q1) store(buf ^ 1);
    __syncthreads();
  };
  for (int q = q0; q < q1; q += 2) {
    stage(q, 0);
    if (q + 1 < q1) stage(q + 1, 1);
  }
  if constexpr (kSets == 2) {
    static_assert(F == 1 && sizeof(lds) >= kMats * 16 * 256 * sizeof(float), "the second set's sums fit");
    f32x4* meet = reinterpret_cast<f32x4*>(&lds[0][0]);
#pragma unroll
    for (int m = 0; m < kMats; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f32x4* at = meet + ((m * 4 + e) * 4 + (wave & 3)) * 64 + lane;
        if (set == 1)
          *at = f32x4{acc[m][0][0][4 * e], acc[m][0][0][4 * e + 1], acc[m][0][0][4 * e + 2], acc[m][0][0][4 * e + 3]};
      }
    __syncthreads();
    if (set == 1) return;
#pragma unroll
    for (int m = 0; m < kMats; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x4 x = meet[((m * 4 + e) * 4 + (wave & 3)) * 64 + lane];
#pragma unroll
        for (int z = 0; z < 4; ++z) acc[m][0][0][4 * e + z] += x[z];
      }
  }
#pragma unroll
  for (int i = 0; i < kFM; ++i)
#pragma unroll
    for (int j = 0; j < F; ++j) {
      const int64_t n = n0 + 32 * (wn * F + j) + lane % 32;
      if (n >= p.N) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int m = (int)m0 + 32 * (wm * kFM + i) + 8 * e + 4 * (lane / 32);
        if (m >= p.M) continue;
        float c[2][4] = {};
#pragma unroll
        for (int x = 0; x < kMats; ++x)
#pragma unroll
          for (int z = 0; z < 4; ++z) c[x][z] = acc[x][i][j][4 * e + z];
        if (p.partial) {
          float* at = p.partial + ((int64_t)blockIdx.y * kMats * p.N + n) * p.Mp + m;
          store_partial(at, c[0]);
          if (kGated) store_partial(at + p.N * p.Mp, c[1]);
        } else {
          write_product<float, KIND, 4>(p.out, n, m, p.M, c[0], c[1]);
        }
      }
    }
}

size_t partial_bytes(const Product& p, const ShapeF32& s) {
  return s.splits == 1 ? 0
                       : sizeof(float) * (size_t)s.splits * (p.kind == kProductGated ? 2 : 1) * (size_t)p.N *
                             (size_t)((p.M + 7) / 8 * 8);
}

template <ProductKind KIND, bool AT, bool BT>
void launch_tiles(TileArgs& t, const ShapeF32& s, hipStream_t stream) {
  for (int64_t first = 0; first < s.m_tiles * s.n_tiles; first += kMostTilesF32) {
    t.first = (uint32_t)first;  // of fewer than 2^32 tiles: their results are in memory
    const dim3 grid((unsigned)s.launch_tiles(first), s.splits);
    if (s.f == 2)
      tile_product_f32_kernel<2, AT, BT, KIND><<<grid, s.threads(), 0, stream>>>(t);
    else
      tile_product_f32_kernel<1, AT, BT, KIND><<<grid, s.threads(), 0, stream>>>(t);
  }
}

}  // namespace

size_t product_bytes_f32(const Product& p) { return partial_bytes(p, choose_f32(p, device_cus())); }

dtp_status launch_product_f32(const Product& p, char* workspace, hipStream_t s) {
  const ShapeF32 shape = choose_f32(p, device_cus());
  const int Mp = (p.M + 7) / 8 * 8;
  float* partial = shape.splits > 1 ? (float*)workspace : nullptr;
  if (shape.stream) {
    const StreamArgs a{p.a0, p.a1, p.b, p.lda, p.ldb, p.M, (int)p.N, Mp, p.K, shape.stages, shape.per, shape.splits,
                       partial, p.out};
    launch_stream<float>(p.kind, a, s);
  } else {
    TileArgs t{};
    t.a0 = (const float*)p.a0;
    t.a1 = (const float*)p.a1;
    t.b = (const float*)p.b;
    t.lda = p.lda;
    t.ldb = p.ldb;
    t.K = p.K;
    t.b_seg = p.b_seg;
    t.M = p.M;
    t.Mp = Mp;
    t.segments = p.segments;
    t.N = p.N;
    t.m_tiles = shape.m_tiles;
    t.per = shape.per;
    t.stages = shape.stages;
    t.partial = partial;
    t.out = p.out;
    switch (p.kind) {
      case kProductLinear: launch_tiles<kProductLinear, false, false>(t, shape, s); break;
      case kProductGated: launch_tiles<kProductGated, false, false>(t, shape, s); break;
      case kProductGrad:
        if (p.bt)
          launch_tiles<kProductGrad, true, true>(t, shape, s);
        else
          launch_tiles<kProductGrad, true, false>(t, shape, s);
    }
  }
  DTP_HIP(hipGetLastError());
  if (partial) {
    launch_join<float>(p.kind, partial, shape.splits, p.M, p.N, Mp, p.out, s);
    DTP_HIP(hipGetLastError());
  }
  return DTP_OK;
}

}  // namespace dtp
