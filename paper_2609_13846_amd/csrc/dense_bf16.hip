// The bf16 products of the dense operators.
//
//   tile_product_kernel    tiles through the LDS ring of row_gemm.h, the contraction split over
//                          blocks where there are few tiles
//   stream_product_kernel, join_product_kernel  few tokens, split contractions (dense_stream.h)
//   pad_rows_kernel        copies of operands whose rows are not whole 16-byte pieces
#include <algorithm>

#include "dense_stream.h"
#include "row_gemm.h"

namespace dtp {
namespace {

struct TileArgs {
  const uint16_t *a0, *a1, *b;
  RowContraction k;
  int M, N, Mp;       // Mp: M rounded up to 8, the row of a partial sum
  int nq, per;        // stages (stream: runs of 64 columns) of the contraction, and of a split
  int m_tiles, n_tiles;
  int64_t bytes_a, bytes_b;  // of the operands
  int64_t second_a;          // bytes from a0 to the second segment's matrix
  float* partial;     // [splits][planes][N][Mp], or NULL
  ProductOut out;
};

__device__ __forceinline__ float half_of(const u32x4& v, int e) {
  return __uint_as_float(e % 2 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
}
__device__ __forceinline__ u32x4 pack_whole(const float (&v)[8]) {
  u32x4 o;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
  return o;
}

// 16 bytes at any address; PAST: past the caches.
template <bool PAST, typename T>
__device__ __forceinline__ void put(T* p, const u32x4& v) {
  if constexpr (PAST)
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4_any*>(p));
  else
    *reinterpret_cast<u32x4_any*>(p) = v;
}

// The eight results of a place, from their sums; bias and residual are theirs.
template <ProductKind KIND>
__device__ __forceinline__ u32x4 finish(const ProductOut& o, const float (&c0)[8], const float (&c1)[8],
                                        const u32x4& residual) {
  float v[8];
  if constexpr (KIND == kProductLinear) {  // c0: with the bias
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c0[e];
    if (o.act != DTP_ACT_NONE) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = activate<uint16_t>(o.act, v[e]);
    }
    if (o.residual) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = fmaf(o.alpha, v[e], half_of(residual, e));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= o.alpha;
    }
  } else if constexpr (KIND == kProductGated) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = activate<uint16_t>(o.act, c0[e]) * c1[e];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = o.alpha * c0[e];
  }
  return pack_whole(v);
}

// Lanes r and r + 8 of 16: a keeps its lower eight lanes and takes b's in the upper ones, b the
// other way round: what was 16 rows of a and of b is 8 rows of a and b, and then the other 8.
__device__ __forceinline__ void exchange_rows(u32x4& a, u32x4& b) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int x = (int)a[e], y = (int)b[e];
    a[e] = (uint32_t)__builtin_amdgcn_update_dpp(x, y, 0x128, 0xf, 0xc, false);  // row_ror:8
    b[e] = (uint32_t)__builtin_amdgcn_update_dpp(y, x, 0x128, 0xf, 0x3, false);
  }
}

// Eight consecutive values per lane group of 16, as a lane's lower and upper four: afterwards a holds
// the 16 lower ones of the four groups' 32 and b the upper, four consecutive in each group.
__device__ __forceinline__ void exchange_groups(u32x4& a, u32x4& b) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const auto half = __builtin_amdgcn_permlane16_swap(a[e], b[e], false, false);
    const auto whole = __builtin_amdgcn_permlane32_swap(half[0], half[1], false, false);
    a[e] = whole[0];
    b[e] = whole[1];
  }
}

// One block per CU (256 x 256 tiles; two of 128 x 128, three of 128 x 64), each with a run of items: a
// tile, or a split of its contraction.  Items are numbered so that the ones that run together on an
// XCD share operands.
// ENDS: M need not be a multiple of 8.  (A kernel of its own for the linear epilogue, which has no
// registers for the rows' ends beside the exchange of lines.)
template <int AF, int BF, bool AT, bool BT, ProductKind KIND, bool ENDS>
__global__ void __launch_bounds__(512, AF * BF > 16 ? 2 : 4) tile_product_kernel(TileArgs p) {
  constexpr bool kGated = KIND == kProductGated;
  using Pipe = RowPipe<AF, BF, AT, BT, kGated>;
  constexpr int kTileM = kGated ? Pipe::kHalf : Pipe::kARows, kTileN = Pipe::kBRows;
  constexpr int kPairs = kGated ? AF / 4 : AF / 2;
  // Forward results of the large tiles, which are more than the L2s hold (32 MiB), are written past
  // them, where they would displace the operands: 65,536 x 1,024 x 6,144 729 -> 704 us, a gated block
  // that keeps its pre-activations 950 -> 915.  (Gradients' are not: dx of 16,384 x 4,096 x 1,536
  // took 166 us instead of 161.)
  constexpr bool kPast = AF * BF > 16 && KIND != kProductGrad, kLines = kPast && (kGated || !ENDS);
  __shared__ __attribute__((aligned(16))) uint16_t s0a0[Pipe::kASlot], s0a1[Pipe::kASlot], s0b[Pipe::kBSlot],
      s1a0[Pipe::kASlot], s1a1[Pipe::kASlot], s1b[Pipe::kBSlot];
  const int tiles = p.m_tiles * p.n_tiles;
  auto place = [&](int i, int& m0, int& n0, int& split) __attribute__((always_inline)) {
    split = i / tiles;
    int tm, tn;
    frag_work(i - split * tiles, p.m_tiles, p.n_tiles, 8, tm, tn);
    m0 = tm * kTileM;
    n0 = tn * kTileN;
  };
  auto item = [&](int i) __attribute__((always_inline)) {
    int m0, n0, split;
    place(i, m0, n0, split);
    RowItem it;
    it.first = split * p.per;
    it.n = min(p.per, p.nq - it.first);
    const bool second = it.first >= p.k.per_segment;
    const int64_t in_seg = second ? it.first - p.k.per_segment : it.first;
    const int64_t oa = (AT ? m0 : m0 * (int64_t)p.k.lda) * 2 + in_seg * p.k.step_a;
    const int64_t ob = (BT ? n0 : n0 * (int64_t)p.k.ldb) * 2 + it.first * p.k.step_b + (second ? p.k.jump_b : 0);
    it.a = (const char*)p.a0 + (second ? p.second_a : 0) + oa;
    it.left_a = p.bytes_a - oa;
    it.b = (const char*)p.b + ob;
    it.left_b = p.bytes_b - ob;
    it.columns = p.k.columns - (int)in_seg * kRowStage;
    return it;
  };
  Pipe pipe(p.k);
  auto done = [&](int i) __attribute__((always_inline)) {
    int m0, n0, split;
    place(i, m0, n0, split);
    const int m_lane = m0 + pipe.wm * (kGated ? 8 * AF : 16 * AF) + 8 * (pipe.lane / 16);
    const int n_lane = n0 + pipe.wn * 16 * BF + pipe.lane % 16;
    auto sums = [&](int i, int j, float (&c0)[8], float (&c1)[8]) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        c0[e] = pipe.acc[2 * i + e / 4][j][e % 4];
        c1[e] = kGated ? pipe.acc[kGated ? AF / 2 + 2 * i + e / 4 : 0][j][e % 4] : 0.0f;
      }
    };
    if (p.partial) {
      pipe.settle();
      const int planes = kGated ? 2 : 1;
#pragma unroll
      for (int j = 0; j < BF; ++j)
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
          const int n = n_lane + 16 * j, m = m_lane + 32 * i;
          if (n >= p.N || m >= p.M) continue;
          float c0[8], c1[8];
          sums(i, j, c0, c1);
          float* at = p.partial + ((int64_t)split * planes * p.N + n) * p.Mp + m;
          store_partial(at, c0);
          if (kGated) store_partial(at + (int64_t)p.N * p.Mp, c1);
        }
      return;
    }
    if (ENDS && p.M % 8 != 0 && m0 + kTileM > p.M) {  // rows that end inside a lane's eight
      pipe.settle();
#pragma unroll
      for (int j = 0; j < BF; ++j)
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
          if (n_lane + 16 * j >= p.N) continue;
          float c0[8], c1[8];
          sums(i, j, c0, c1);
          write_product<uint16_t, KIND, 8>(p.out, n_lane + 16 * j, m_lane + 32 * i, p.M, c0, c1);
        }
      return;
    }
    // results a row at a time, the next row's residual on its way beside this one's writes
    constexpr bool kLinear = KIND == kProductLinear;
    u32x4 bias[kPairs] = {}, residual[2][kPairs] = {};
    if (kLinear && p.out.bias) {
#pragma unroll
      for (int i = 0; i < kPairs; ++i)
        if (m_lane + 32 * i < p.M) bias[i] = *reinterpret_cast<const u32x4*>((const uint16_t*)p.out.bias + m_lane + 32 * i);
    }
    auto fetch = [&](int j) __attribute__((always_inline)) {
      if (!kLinear || !p.out.residual || n_lane + 16 * j >= p.N) return;
#pragma unroll
      for (int i = 0; i < kPairs; ++i)
        if (m_lane + 32 * i < p.M)
          residual[j % 2][i] = *reinterpret_cast<const u32x4_any*>((const uint16_t*)p.out.residual +
                                                               (int64_t)(n_lane + 16 * j) * p.M + m_lane + 32 * i);
    };
    fetch(0);
    // Results past the caches go in whole 128-byte lines, eight rows at a time: the lanes' values
    // change places first.  (In halves and quarters of lines memory took 15 to 35% more bytes:
    // 918 us for a gated block over 65,536 tokens that keeps its pre-activations, and 867; 877 for
    // 65,536 x 1,024 x 6,144 with bias and residual, and 837.)
    const int r8 = pipe.lane % 8, upper = pipe.lane % 16 / 8, group = pipe.lane / 16;
    const int m_wave = m_lane - 8 * group, n_wave = n_lane - pipe.lane % 16;
    auto store_kept = [&](int plane, int i, int j, const float (&c)[8]) __attribute__((always_inline)) {
      if constexpr (kLines) {
        u32x4 x, y;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = __float_as_uint(c[e]);
          y[e] = __float_as_uint(c[4 + e]);
        }
        exchange_groups(x, y);
        exchange_rows(x, y);
        const int m = m_wave + 32 * i + 16 * upper + 4 * group;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int n = n_wave + 16 * j + 8 * h + r8;
          if (n >= p.N || m >= p.M) continue;
          float* at = p.out.pre + ((int64_t)n * (kGated ? 2 : 1) + plane) * p.M + m;
          put<kPast>(at, h ? y : x);
        }
      } else {
        const int n = n_lane + 16 * j, m = m_lane + 32 * i;
        if (n >= p.N || m >= p.M) return;
        float* at = p.out.pre + ((int64_t)n * (kGated ? 2 : 1) + plane) * p.M + m;
        put<kPast>(at, u32x4{__float_as_uint(c[0]), __float_as_uint(c[1]), __float_as_uint(c[2]), __float_as_uint(c[3])});
        put<kPast>(at + 4, u32x4{__float_as_uint(c[4]), __float_as_uint(c[5]), __float_as_uint(c[6]), __float_as_uint(c[7])});
      }
    };
#pragma unroll
    for (int j = 0; j < BF; ++j) {
      if (j + 1 < BF) fetch(j + 1);
      if (j == 0) pipe.settle();
      u32x4 out[kPairs];
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const int n = n_lane + 16 * j, m = m_lane + 32 * i;
        if (!kLines && (n >= p.N || m >= p.M)) continue;
        float c0[8], c1[8];
        sums(i, j, c0, c1);
        if (kLinear) {
#pragma unroll
          for (int e = 0; e < 8; ++e) c0[e] += half_of(bias[i], e);
        }
        if (KIND != kProductGrad && p.out.pre) {
          store_kept(0, i, j, c0);
          if (kGated) store_kept(1, i, j, c1);
        }
        out[i] = finish<KIND>(p.out, c0, c1, residual[j % 2][i]);
        if constexpr (!kLines) {
          uint16_t *const y1 = (uint16_t*)p.out.y, *const y2 = (uint16_t*)p.out.y2;
          const bool second = KIND == kProductGrad && n >= p.out.n_split;
          const int64_t row = second ? n - p.out.n_split : n;
          if (KIND == kProductGrad && row >= p.out.n_keep) continue;
          put<kPast>((second ? y2 : y1) + row * p.M + m, out[i]);
        }
      }
      if constexpr (kLines) {
#pragma unroll
        for (int i = 0; i < kPairs; i += 2) {
          exchange_rows(out[i], out[i + 1]);
          const int m = m_wave + 32 * (i + upper) + 8 * group;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int n = n_wave + 16 * j + 8 * h + r8;
            if (n < p.N && m < p.M) put<kPast>((uint16_t*)p.out.y + (int64_t)n * p.M + m, out[i + h]);
          }
        }
      }
    }
  };
  const int items = tiles * ((p.nq + p.per - 1) / p.per);
  pipe.run({s0a0, s0a1, s0b}, {s1a0, s1a1, s1b}, blockIdx.x, items, gridDim.x, item, done);
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

// ---------------------------------------------------------------------------- launches
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// Rows and row length of an operand as it lies in memory.
struct Lines {
  int64_t rows, n;
  bool pad;
  size_t bytes() const { return pad ? up256(2 * (size_t)(rows * pad32(n))) : 0; }
};
Lines lines_a(const Product& p) { return {p.at ? p.K : p.M, p.at ? p.M : p.K, p.lda % 8 != 0 && !streams_bf16(p)}; }
Lines lines_b(const Product& p) { return {p.bt ? p.K : p.N, p.bt ? p.N : p.K, p.ldb % 8 != 0 && !streams_bf16(p)}; }

size_t partial_bytes(const Product& p, const ShapeBf16& s) {
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
void launch_tiles(TileArgs& t, const ShapeBf16& s, hipStream_t stream) {
  if (KIND == kProductGated) {
    t.k.half_a = (const char*)t.a1 - (const char*)t.a0;
  } else {
    t.k.half_a = t.k.half_left = (kTilesBf16[s.tile].m / 2) * (AT ? 1 : (int64_t)t.k.lda);  // 8 AF rows
  }
  const int items = t.m_tiles * t.n_tiles * s.splits, grid = std::min(items, kTilesBf16[s.tile].per_cu * device_cus());
  auto launch = [&](auto ends) {
    constexpr bool kEnds = decltype(ends)::value;
    if (s.tile == 0)
      tile_product_kernel<8, 4, AT, BT, KIND, kEnds><<<grid, 512, 0, stream>>>(t);
    else if (s.tile == 1)
      tile_product_kernel<4, 2, AT, BT, KIND, kEnds><<<grid, 512, 0, stream>>>(t);
    else
      tile_product_kernel<4, 1, AT, BT, KIND, kEnds><<<grid, 512, 0, stream>>>(t);
  };
  if constexpr (KIND == kProductLinear) {
    if (t.M % 8 == 0) return launch(std::false_type());
  }
  launch(std::true_type());
}

}  // namespace

size_t product_bytes_bf16(const Product& p) {
  const Lines a = lines_a(p), b = lines_b(p);
  const bool two = p.kind == kProductGated || p.segments == 2;
  return (two ? 2 : 1) * a.bytes() + b.bytes() + partial_bytes(p, choose_bf16(p, device_cus()));
}

dtp_status launch_product_bf16(const Product& p, char* workspace, hipStream_t s) {
  const ShapeBf16 shape = choose_bf16(p, device_cus());
  const Lines la = lines_a(p), lb = lines_b(p);
  TileArgs t{};
  t.a0 = padded(p.a0, la, workspace, s);
  t.a1 = padded(p.a1, la, workspace, s);
  t.b = padded(p.b, lb, workspace, s);
  DTP_HIP(hipGetLastError());
  t.k.lda = (uint32_t)(la.pad ? pad32(la.n) : p.lda);
  t.k.ldb = (uint32_t)(lb.pad ? pad32(lb.n) : p.ldb);
  t.bytes_a = 2 * la.rows * (int64_t)t.k.lda;
  t.bytes_b = 2 * lb.rows * (int64_t)t.k.ldb;
  t.k.step_a = 2 * kRowStage * (p.at ? (int64_t)t.k.lda : 1);
  t.k.step_b = 2 * kRowStage * (p.bt ? (int64_t)t.k.ldb : 1);
  t.k.per_segment = shape.nq / p.segments;
  t.k.columns = (int)p.K;
  if (p.segments == 2) {
    t.second_a = (const char*)t.a1 - (const char*)t.a0;
    t.k.jump_a = t.second_a - t.k.per_segment * t.k.step_a;
    t.k.jump_b = 2 * p.b_seg - t.k.per_segment * t.k.step_b;
  }
  t.M = p.M;
  t.N = (int)p.N;
  t.Mp = (p.M + 7) / 8 * 8;
  t.nq = shape.nq;
  t.per = shape.per;
  t.partial = shape.splits > 1 ? (float*)workspace : nullptr;
  t.out = p.out;
  if (shape.stream) {
    StreamArgs r{t.a0, t.a1, t.b, t.k.lda, t.k.ldb, t.M, t.N, t.Mp, p.K, shape.nq, shape.per, shape.splits, t.partial, t.out};
    launch_stream<uint16_t>(p.kind, r, s);
  } else {
    t.m_tiles = (int)(((int64_t)(p.kind == kProductGated ? 2 : 1) * p.M + kTilesBf16[shape.tile].m - 1) / kTilesBf16[shape.tile].m);
    t.n_tiles = (int)((p.N + kTilesBf16[shape.tile].n - 1) / kTilesBf16[shape.tile].n);
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
    launch_join<uint16_t>(p.kind, t.partial, shape.splits, t.M, t.N, t.Mp, t.out, s);
    DTP_HIP(hipGetLastError());
  }
  return DTP_OK;
}

}  // namespace dtp
