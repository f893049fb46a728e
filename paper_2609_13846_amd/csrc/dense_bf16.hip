// The bf16 products of the dense operators.
//
//   tile_product_kernel    tiles through the LDS ring of row_gemm.h, the contraction split over
//                          blocks where there are few tiles
//   stream_product_kernel  few tokens: the weights streamed once, straight into registers
//   join_product_kernel    the sum of a split contraction's parts, with the product's epilogue
//   pad_rows_kernel        copies of operands whose rows are not whole 16-byte pieces
#include <algorithm>

#include "dense.h"
#include "row_gemm.h"

namespace dtp {
namespace {

constexpr int kCus = 256;

struct TileArgs {
  const uint16_t *a0, *a1, *b;
  int64_t lda, ldb;
  int M, N, Mp;       // Mp: M rounded up to 8, the row of a partial sum
  int64_t K;          // columns per segment
  int nq_seg, nq;     // stages per segment, and of the whole contraction
  int per;            // stages per split
  int m_tiles, n_tiles;
  uint32_t b_jump;
  float* partial;     // [splits][planes][N][Mp], or NULL
  ProductOut out;
};

template <int W>
__device__ __forceinline__ void store_partial(float* p, const float (&v)[W]) {
#pragma unroll
  for (int i = 0; i < W; i += 4) *reinterpret_cast<f32x4*>(p + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
}

template <int AF, int BF, bool AT, bool BT, ProductKind KIND>
__global__ void __launch_bounds__(512, AF * BF > 16 ? 2 : 4) tile_product_kernel(TileArgs p) {
  constexpr bool kGated = KIND == kProductGated;
  using Pipe = RowPipe<AF, BF, AT, BT, kGated>;
  constexpr int kTileM = kGated ? Pipe::kARows / 2 : Pipe::kARows, kTileN = Pipe::kBRows;
  __shared__ __attribute__((aligned(16))) uint16_t s0[Pipe::kSlot], s1[Pipe::kSlot], s2[Pipe::kSlot], s3[Pipe::kSlot];
  int tm, tn;
  frag_work(blockIdx.x, p.m_tiles, p.n_tiles, 8, tm, tn);
  const int m0 = tm * kTileM, n0 = tn * kTileN;
  const int q0 = blockIdx.y * p.per, q1 = min(q0 + p.per, p.nq);
  const bool rebase = p.nq == p.nq_seg;  // one segment: pointers at the split's first stage
  const int64_t first = rebase ? (int64_t)q0 * 32 : 0;
  auto operand = [&](const uint16_t* x, const uint16_t* x2, int64_t ld, bool across, int row, int64_t rows) {
    const int64_t o = across ? first * ld + row : (int64_t)row * ld + first;
    const int64_t left = 2 * ((across ? p.K : rows) * ld - o);
    return RowOperand{x + o, x2 ? x2 + o : nullptr, ld, left < (int64_t)kRowRange ? (uint32_t)left : kRowRange};
  };
  Pipe pipe(operand(p.a0, p.a1, p.lda, AT, m0, p.M), operand(p.b, nullptr, p.ldb, BT, n0, p.N), p.b_jump);
  pipe.contract(s0, s1, s2, s3, q0, q1, p.nq_seg, p.K, rebase ? q0 : 0);

  constexpr int kPairs = kGated ? AF / 4 : AF / 2;
  const int planes = kGated ? 2 : 1;
  const int m_lane = m0 + pipe.wm * (kGated ? 8 * AF : 16 * AF) + 8 * (pipe.lane / 16);
#pragma unroll
  for (int j = 0; j < BF; ++j) {
    const int n = n0 + pipe.wn * 16 * BF + 16 * j + pipe.lane % 16;
    if (n >= p.N) continue;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const int m = m_lane + 32 * i;
      float c0[8], c1[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        c0[e] = pipe.acc[2 * i + e / 4][j][e % 4];
        c1[e] = kGated ? pipe.acc[kGated ? AF / 2 + 2 * i + e / 4 : 0][j][e % 4] : 0.0f;
      }
      if (p.partial) {
        if (m >= p.M) continue;
        float* at = p.partial + ((int64_t)blockIdx.y * planes * p.N + n) * p.Mp + m;
        store_partial(at, c0);
        if (kGated) store_partial(at + (int64_t)p.N * p.Mp, c1);
      } else {
        write_product<uint16_t, KIND, 8>(p.out, n, m, p.M, c0, c1);
      }
    }
  }
}

// Few tokens (at most 16 TF): the time is that of reading the weights once.  A block takes 16
// features (gated: 16 of each projection), its eight wavefronts deal out the columns in runs of
// 64, and their sums meet in LDS.  Weights go straight into the matrix instruction's registers:
// lane l reads 32 bytes of row l % 16, columns 16 (l / 16) of the run on, and the tokens' lanes
// read the same columns, so any order of columns is as good as another.
template <int TF, ProductKind KIND>
__global__ void __launch_bounds__(512) stream_product_kernel(TileArgs p) {
  constexpr bool kGated = KIND == kProductGated;
  constexpr int kMats = kGated ? 2 : 1, kUnroll = TF > 1 ? 2 : 4;
  __shared__ f32x4 sums[8][kMats * TF][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int r = lane % 16, g = lane / 16;
  const int m0 = blockIdx.x * 16, m = min(m0 + r, p.M - 1);
  const uint16_t* a[kMats];
  a[0] = p.a0 + (int64_t)m * p.lda + 16 * g;
  if constexpr (kGated) a[1] = p.a1 + (int64_t)m * p.lda + 16 * g;
  const uint16_t* b[TF];
#pragma unroll
  for (int t = 0; t < TF; ++t) b[t] = p.b + (int64_t)min(16 * t + r, p.N - 1) * p.ldb + 16 * g;
  f32x4 acc[kMats][TF] = {};
  const int c0 = blockIdx.y * p.per, c1 = min(c0 + p.per, p.nq);  // runs
  const int whole = min(c1, (int)(p.K / 64));
  auto load = [](const uint16_t* q) { return *reinterpret_cast<const bf16x8*>(q); };
  auto run = [&](auto n, int c) __attribute__((always_inline)) {
    constexpr int N = decltype(n)::value;
    bf16x8 fa[N][kMats][2], fb[N][TF][2];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int k = (c + 8 * u) * 64;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < kMats; ++i) fa[u][i][h] = load(a[i] + k + 8 * h);
#pragma unroll
        for (int t = 0; t < TF; ++t) fb[u][t][h] = load(b[t] + k + 8 * h);
      }
    }
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < kMats; ++i)
#pragma unroll
          for (int t = 0; t < TF; ++t)
            acc[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[u][i][h], fb[u][t][h], acc[i][t], 0, 0, 0);
  };
  int c = c0 + wave;
  for (; c + 8 * (kUnroll - 1) < whole; c += 8 * kUnroll) run(std::integral_constant<int, kUnroll>(), c);
  for (; c < whole; c += 8) run(std::integral_constant<int, 1>(), c);
  if (c < c1) {  // the run that the columns end in
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = c * 64 + 8 * h;
      const bool in = k + 16 * g < p.K;
      bf16x8 fa[kMats] = {};
#pragma unroll
      for (int i = 0; i < kMats; ++i)
        if (in) fa[i] = load(a[i] + k);
#pragma unroll
      for (int t = 0; t < TF; ++t) {
        bf16x8 fb = {};
        if (in) fb = load(b[t] + k);
#pragma unroll
        for (int i = 0; i < kMats; ++i) acc[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[i], fb, acc[i][t], 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kMats; ++i)
#pragma unroll
    for (int t = 0; t < TF; ++t) sums[wave][i * TF + t][lane] = acc[i][t];
  __syncthreads();
  const int idx = threadIdx.x;
  if (idx >= 32 * TF) return;
  const int half = idx % 2, n = idx / 2, mm = m0 + 8 * half;
  if (n >= p.N || mm >= p.M) return;
  float v[2][8] = {};
#pragma unroll
  for (int i = 0; i < kMats; ++i)
#pragma unroll
    for (int w = 0; w < 8; ++w)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] += sums[w][i * TF + n / 16][(2 * half + e / 4) * 16 + n % 16][e % 4];
  if (p.partial) {
    float* at = p.partial + ((int64_t)blockIdx.y * kMats * p.N + n) * p.Mp + mm;
    store_partial(at, v[0]);
    if (kGated) store_partial(at + (int64_t)p.N * p.Mp, v[1]);
  } else {
    write_product<uint16_t, KIND, 8>(p.out, n, mm, p.M, v[0], v[1]);
  }
}

template <ProductKind KIND>
__global__ void __launch_bounds__(256) join_product_kernel(const float* __restrict__ partial, int splits, int M, int N,
                                                           int Mp, ProductOut out) {
  constexpr int kPlanes = KIND == kProductGated ? 2 : 1;
  const int pieces = Mp / 8;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)N * pieces; i += (int64_t)gridDim.x * 256) {
    const int64_t n = i / pieces;
    const int m = (int)(i - n * pieces) * 8;
    float v[2][8] = {};
    for (int s = 0; s < splits; ++s)
#pragma unroll
      for (int pl = 0; pl < kPlanes; ++pl) {
        const f32x4* at = reinterpret_cast<const f32x4*>(partial + (((int64_t)s * kPlanes + pl) * N + n) * Mp + m);
        const f32x4 lo = at[0], hi = at[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[pl][e] += lo[e];
          v[pl][4 + e] += hi[e];
        }
      }
    write_product<uint16_t, KIND, 8>(out, n, m, M, v[0], v[1]);
  }
}

// out[r][0 .. ld) = in[r][0 .. n), zeros behind.
__global__ void __launch_bounds__(256) pad_rows_kernel(const uint16_t* __restrict__ in, int64_t rows, int n, int ld,
                                                       uint16_t* __restrict__ out) {
  const int pieces = ld / 8;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * pieces; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / pieces;
    const int c = (int)(i - r * pieces) * 8;
    u32x4 v = {};
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < n) v[e / 2] |= (uint32_t)in[r * n + c + e] << (16 * (e % 2));
    *reinterpret_cast<u32x4*>(out + r * ld + c) = v;
  }
}

// ---------------------------------------------------------------------------- plan
struct Shape {
  bool stream = false;
  int tile = 256;      // rows and columns of a tile
  int splits = 1, per = 0, nq = 0, nq_seg = 0;
};

Shape choose(const Product& p) {
  Shape s;
  const bool gated = p.kind == kProductGated;
  if (!p.at && !p.bt && p.N <= 64) {
    s.stream = true;
    s.nq = s.nq_seg = (int)((p.K + 63) / 64);
    const int rows = (p.M + 15) / 16;
    int splits = 1;
    while (rows * splits < kCus / 2 && s.nq / (splits * 2) >= 16) splits *= 2;
    s.per = (s.nq + splits - 1) / splits;
  } else {
    s.nq_seg = (int)((p.K + 31) / 32);
    s.nq = s.nq_seg * p.segments;
    auto tiles = [&](int t) { return ((int64_t)(gated ? 2 : 1) * p.M + t - 1) / t * ((p.N + t - 1) / t); };
    s.tile = tiles(256) >= 192 ? 256 : 128;
    const int64_t n = tiles(s.tile), room = s.tile == 256 ? kCus : 2 * kCus;
    const int64_t splits = std::max<int64_t>(1, std::min<int64_t>({room / n, s.nq / 8, 16}));
    s.per = (int)((s.nq + splits - 1) / splits);
    // what a block reaches of an operand across has 31 bits
    if (p.at || p.bt) {
      const int64_t line = 64 * std::max(p.at ? p.lda : 0, p.bt ? p.ldb : 0);
      if (p.segments == 1) s.per = (int)std::min<int64_t>(s.per, (int64_t)(kRowRange - 1) / line);
    }
  }
  s.splits = (s.nq + s.per - 1) / s.per;
  return s;
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }
int64_t pad32(int64_t n) { return (n + 31) / 32 * 32; }

// Rows and row length of an operand as it lies in memory.
struct Lines {
  int64_t rows, n;
  bool pad;
  size_t bytes() const { return pad ? up256(2 * (size_t)(rows * pad32(n))) : 0; }
};
Lines lines_a(const Product& p) { return {p.at ? p.K : p.M, p.at ? p.M : p.K, p.lda % 8 != 0}; }
Lines lines_b(const Product& p) { return {p.bt ? p.K : p.N, p.bt ? p.N : p.K, p.ldb % 8 != 0}; }

size_t partial_bytes(const Product& p, const Shape& s) {
  if (s.splits == 1) return 0;
  return sizeof(float) * (size_t)s.splits * (p.kind == kProductGated ? 2 : 1) * (size_t)p.N * ((p.M + 7) / 8 * 8);
}

const uint16_t* padded(const void* in, const Lines& l, char*& at, hipStream_t s) {
  if (!l.pad || in == nullptr) return (const uint16_t*)in;
  uint16_t* out = (uint16_t*)at;
  const int ld = (int)pad32(l.n);
  const int64_t threads = l.rows * (ld / 8);
  pad_rows_kernel<<<(unsigned)std::min<int64_t>((threads + 255) / 256, 16384), 256, 0, s>>>((const uint16_t*)in, l.rows,
                                                                                           (int)l.n, ld, out);
  at += l.bytes();
  return out;
}

template <ProductKind KIND, bool AT, bool BT>
void launch_tiles(const TileArgs& t, const Shape& s, hipStream_t stream) {
  const dim3 grid(t.m_tiles * t.n_tiles, s.splits);
  if (s.tile == 256)
    tile_product_kernel<8, 4, AT, BT, KIND><<<grid, 512, 0, stream>>>(t);
  else
    tile_product_kernel<4, 2, AT, BT, KIND><<<grid, 512, 0, stream>>>(t);
}

template <ProductKind KIND>
void launch_stream(const TileArgs& t, const Shape& s, hipStream_t stream) {
  const dim3 grid((t.M + 15) / 16, s.splits);
  if (t.N <= 16)
    stream_product_kernel<1, KIND><<<grid, 512, 0, stream>>>(t);
  else if (t.N <= 32)
    stream_product_kernel<2, KIND><<<grid, 512, 0, stream>>>(t);
  else
    stream_product_kernel<4, KIND><<<grid, 512, 0, stream>>>(t);
}

template <ProductKind KIND>
void launch_join(const TileArgs& t, const Shape& s, hipStream_t stream) {
  const int64_t threads = (int64_t)t.N * (t.Mp / 8);
  join_product_kernel<KIND><<<(unsigned)std::min<int64_t>((threads + 255) / 256, 8192), 256, 0, stream>>>(
      t.partial, s.splits, t.M, t.N, t.Mp, t.out);
}

}  // namespace

size_t product_bytes_bf16(const Product& p) {
  const Lines a = lines_a(p), b = lines_b(p);
  const bool two = p.kind == kProductGated || p.segments == 2;
  return (two ? 2 : 1) * a.bytes() + b.bytes() + partial_bytes(p, choose(p));
}

dtp_status launch_product_bf16(const Product& p, char* workspace, hipStream_t s) {
  const Shape shape = choose(p);
  const Lines la = lines_a(p), lb = lines_b(p);
  TileArgs t{};
  t.a0 = padded(p.a0, la, workspace, s);
  t.a1 = padded(p.a1, la, workspace, s);
  t.b = padded(p.b, lb, workspace, s);
  DTP_HIP(hipGetLastError());
  t.lda = la.pad ? pad32(la.n) : p.lda;
  t.ldb = lb.pad ? pad32(lb.n) : p.ldb;
  t.M = p.M;
  t.N = (int)p.N;
  t.Mp = (p.M + 7) / 8 * 8;
  t.K = p.K;
  t.nq_seg = shape.nq_seg;
  t.nq = shape.nq;
  t.per = shape.per;
  t.b_jump = (uint32_t)(2 * p.b_seg);
  t.partial = shape.splits > 1 ? (float*)workspace : nullptr;
  t.out = p.out;
  if (shape.stream) {
    p.kind == kProductGated ? launch_stream<kProductGated>(t, shape, s) : launch_stream<kProductLinear>(t, shape, s);
  } else {
    t.m_tiles = (int)(((int64_t)(p.kind == kProductGated ? 2 : 1) * p.M + shape.tile - 1) / shape.tile);
    t.n_tiles = (int)((p.N + shape.tile - 1) / shape.tile);
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
  if (t.partial) {
    switch (p.kind) {
      case kProductLinear: launch_join<kProductLinear>(t, shape, s); break;
      case kProductGated: launch_join<kProductGated>(t, shape, s); break;
      case kProductGrad: launch_join<kProductGrad>(t, shape, s); break;
    }
    DTP_HIP(hipGetLastError());
  }
  return DTP_OK;
}

}  // namespace dtp
