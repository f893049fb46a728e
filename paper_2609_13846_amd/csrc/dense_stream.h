// Products of few tokens, and the sum of a split contraction's parts (bf16 and fp32).
#pragma once

#include <algorithm>

#include "dense.h"

namespace dtp {

struct StreamArgs {
  const void *a0, *a1, *b;
  int64_t lda, ldb;
  int M, N, Mp;    // Mp: M rounded up to 8, the row of a partial sum
  int64_t K;
  int runs, per;   // runs of columns in all, and per split
  int splits;
  float* partial;  // [splits][planes][N][Mp], or NULL
  ProductOut out;
};

#ifdef __HIPCC__

namespace {

template <int W>
__device__ __forceinline__ void store_partial(float* p, const float (&v)[W]) {
#pragma unroll
  for (int i = 0; i < W; i += 4) *reinterpret_cast<f32x4*>(p + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
}

// 16 bytes of a row, and the products of two of them: a lane's elements are of the same columns in
// both operands, so that it does not matter which of the instruction's columns each is.
template <typename S>
struct Piece;
template <>
struct Piece<uint16_t> {
  typedef bf16x8 V;
  __device__ static __forceinline__ V load(const uint16_t* p) {
    return __builtin_bit_cast(V, (u32x4)*reinterpret_cast<const u32x4_any*>(p));
  }
  __device__ static __forceinline__ V load_some(const uint16_t* p, int n) {
    u32x4 v = {};
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) v[e / 2] |= (uint32_t)p[e] << (16 * (e % 2));
    return __builtin_bit_cast(V, v);
  }
  __device__ static __forceinline__ f32x4 multiply(const V& a, const V& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Piece<float> {
  typedef f32x4 V;
  __device__ static __forceinline__ V load(const float* p) { return *reinterpret_cast<const f32x4_any*>(p); }
  __device__ static __forceinline__ V load_some(const float* p, int n) {
    V v = {};
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < n) v[e] = p[e];
    return v;
  }
  __device__ static __forceinline__ f32x4 multiply(const V& a, const V& b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
};

// At most 16 tokens: the time is that of reading the weights once.  A block takes 16 features (gated:
// of each projection), its eight wavefronts deal out the columns in runs of 128 bytes a
// row, and their sums meet in LDS.  Weights and tokens go straight into the matrix instruction's
// registers: lane l reads 32 bytes of row l % 16, from byte 32 (l / 16) of the run on.  The loads
// of the next group of runs are in flight while this one's are multiplied.  One token through a gated
// block of 4,096 x 14,336: 43 us, 5.4 TB/s.
template <typename S, ProductKind KIND>
__global__ void __launch_bounds__(512, 4) stream_product_kernel(StreamArgs p) {
  using P = Piece<S>;
  using V = typename P::V;
  constexpr bool kGated = KIND == kProductGated;
  constexpr int kMats = kGated ? 2 : 1;
  constexpr int kWide = 16 / sizeof(S), kRun = 8 * kWide;  // columns of a piece, and of a run
  constexpr int kGroup = 2;                                // runs in flight beside those multiplied
  __shared__ f32x4 sums[8][kMats][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int r = lane % 16, g = lane / 16;
  const int m0 = blockIdx.x * 16, m = min(m0 + r, p.M - 1);
  const S* a[kMats];
#pragma unroll
  for (int i = 0; i < kMats; ++i) a[i] = (const S*)(i ? p.a1 : p.a0) + (int64_t)m * p.lda + 2 * kWide * g;
  const S* b = (const S*)p.b + (int64_t)min(r, p.N - 1) * p.ldb + 2 * kWide * g;
  f32x4 acc[kMats] = {};
  const int c0 = blockIdx.y * p.per, c1 = min(c0 + p.per, p.runs);
  const int whole = min(c1, (int)(p.K / kRun));
  struct Group {
    V a[kGroup][kMats][2], b[kGroup][2];
  };
  Group x, y;
  auto fetch = [&](Group& f, int c) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kGroup; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t k = (int64_t)(c + 8 * u) * kRun + kWide * h;
#pragma unroll
        for (int i = 0; i < kMats; ++i) f.a[u][i][h] = P::load(a[i] + k);
        f.b[u][h] = P::load(b + k);
      }
  };
  auto multiply = [&](const Group& f) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kGroup; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < kMats; ++i) acc[i] = P::multiply(f.a[u][i][h], f.b[u][h], acc[i]);
  };
  constexpr int kStep = 8 * kGroup;  // runs that a group of all wavefronts covers
  int c = c0 + wave;
  const int groups = max(0, (whole - c + 7) / 8 / kGroup);  // whole ones of this wavefront
  if (groups > 0) fetch(x, c);
  for (int q = 0; q < groups; q += 2) {
    if (q + 1 < groups) fetch(y, c + kStep);
    __builtin_amdgcn_sched_barrier(0);
    multiply(x);
    if (q + 1 >= groups) break;
    if (q + 2 < groups) fetch(x, c + 2 * kStep);
    __builtin_amdgcn_sched_barrier(0);
    multiply(y);
    c += 2 * kStep;
  }
  for (c = c0 + wave + groups * kStep; c < c1; c += 8)  // single runs, and the one that the columns end in
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t k = (int64_t)c * kRun + kWide * h;
      V xb = {}, xa[kMats] = {};
      const int64_t left = p.K - k - 2 * kWide * g;
      if (left >= kWide) {
        xb = P::load(b + k);
#pragma unroll
        for (int i = 0; i < kMats; ++i) xa[i] = P::load(a[i] + k);
      } else if (left > 0) {
        xb = P::load_some(b + k, (int)left);
#pragma unroll
        for (int i = 0; i < kMats; ++i) xa[i] = P::load_some(a[i] + k, (int)left);
      }
#pragma unroll
      for (int i = 0; i < kMats; ++i) acc[i] = P::multiply(xa[i], xb, acc[i]);
    }
#pragma unroll
  for (int i = 0; i < kMats; ++i) sums[wave][i][lane] = acc[i];
  __syncthreads();
  // a thread per W features of a token; lane 16 (m / 4) + n of a fragment holds rows m .. m + 3
  constexpr int W = Elem<S>::kWide, kPieces = 16 / W;
  const int n = threadIdx.x / kPieces, row = threadIdx.x % kPieces * W, mm = m0 + row;
  if (n >= p.N || mm >= p.M) return;
  float v[2][W] = {};
#pragma unroll
  for (int i = 0; i < kMats; ++i)
#pragma unroll
    for (int w = 0; w < 8; ++w)
#pragma unroll
      for (int e = 0; e < W; e += 4) {
        const f32x4 s = sums[w][i][(row + e) / 4 * 16 + n];
#pragma unroll
        for (int z = 0; z < 4; ++z) v[i][e + z] += s[z];
      }
  if (p.partial) {
    float* at = p.partial + ((int64_t)blockIdx.y * kMats * p.N + n) * p.Mp + mm;
    store_partial(at, v[0]);
    if (kGated) store_partial(at + (int64_t)p.N * p.Mp, v[1]);
  } else {
    write_product<S, KIND, W>(p.out, n, mm, p.M, v[0], v[1]);
  }
}

// The sums of a split contraction's parts, in order.  Eight parts' loads at a time, where a result has one
// plane: few threads have nothing else to wait beside (16 x 14,336 x 4,096, 16 parts: 6.4 -> 4.6 us here,
// 30.2 -> 28.0 in all; 64 tokens 31.2 -> 31.8; of two planes four parts at a time took 6% longer in all).
template <typename S, ProductKind KIND>
__global__ void __launch_bounds__(256) join_product_kernel(const float* __restrict__ partial, int splits, int M, int64_t N,
                                                           int Mp, ProductOut out) {
  constexpr int kPlanes = KIND == kProductGated ? 2 : 1, W = Elem<S>::kWide, kAhead = kPlanes > 1 ? 1 : 8;
  const int pieces = Mp / W;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < N * pieces; i += (int64_t)gridDim.x * 256) {
    const int64_t n = i / pieces;
    const int m = (int)(i - n * pieces) * W;
    float v[2][W] = {};
#pragma unroll kAhead
    for (int s = 0; s < splits; ++s)
#pragma unroll
      for (int pl = 0; pl < kPlanes; ++pl) {
        const f32x4* at = reinterpret_cast<const f32x4*>(partial + (((int64_t)s * kPlanes + pl) * N + n) * Mp + m);
#pragma unroll
        for (int e = 0; e < W; e += 4) {
          const f32x4 x = at[e / 4];
#pragma unroll
          for (int z = 0; z < 4; ++z) v[pl][e + z] += x[z];
        }
      }
    write_product<S, KIND, W>(out, n, m, M, v[0], v[1]);
  }
}

template <typename S, ProductKind KIND>
void launch_stream_kind(const StreamArgs& a, hipStream_t s) {
  stream_product_kernel<S, KIND><<<dim3((a.M + 15) / 16, a.splits), 512, 0, s>>>(a);
}

template <typename S>
void launch_stream(ProductKind kind, const StreamArgs& a, hipStream_t s) {
  if (kind == kProductGated)
    launch_stream_kind<S, kProductGated>(a, s);
  else
    launch_stream_kind<S, kProductLinear>(a, s);
}

template <typename S>
void launch_join(ProductKind kind, const float* partial, int splits, int M, int64_t N, int Mp, const ProductOut& out,
                 hipStream_t s) {
  const unsigned blocks = (unsigned)std::min<int64_t>((N * (Mp / Elem<S>::kWide) + 255) / 256, 8192);
  if (kind == kProductLinear)
    join_product_kernel<S, kProductLinear><<<blocks, 256, 0, s>>>(partial, splits, M, N, Mp, out);
  else if (kind == kProductGated)
    join_product_kernel<S, kProductGated><<<blocks, 256, 0, s>>>(partial, splits, M, N, Mp, out);
  else
    join_product_kernel<S, kProductGrad><<<blocks, 256, 0, s>>>(partial, splits, M, N, Mp, out);
}

}  // namespace

#endif  // __HIPCC__

}  // namespace dtp
