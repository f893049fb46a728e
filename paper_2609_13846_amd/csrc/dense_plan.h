// The products of a dense decoder layer (linear and gated operators) on the host: what each
// computes, and the tile and splits that it is launched with.  No GPU is needed here.
//
// Every product is  C[n][m] = sum_k A(m, k) B(n, k),  m contiguous in the results:
//   forward   m output feature, n token,          k input feature   (A = W, B = x)
//   dx        m input feature,  n token,          k output feature  (A = W transposed, B = dz)
//   dW        m input feature,  n output feature, k token           (A = x, B = dz transposed)
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

#include "dtp.h"

namespace dtp {

constexpr int kRowStage = 64;  // columns per stage: bf16 tiles
constexpr int kStageF32 = 32;  // fp32 tiles
constexpr int kStreamTokens = 16;

enum ProductKind {
  kProductLinear,  // y = residual + alpha act(C + bias), C + bias kept in `pre`
  kProductGated,   // two products with one B: y = act(C0) C1, both kept in `pre`
  kProductGrad,    // y = alpha C; rows n from n_split on go to y2
};

// Where an element (n, m) of a product goes, and what is done to it on the way.
struct ProductOut {
  void* y = nullptr;
  void* y2 = nullptr;
  const void* bias = nullptr;      // [M]
  const void* residual = nullptr;  // [N][M]
  float* pre = nullptr;            // linear [N][M], gated [N][2][M]
  float alpha = 1.0f;
  int act = DTP_ACT_NONE;
  int64_t n_split = INT64_MAX;  // gradient rows: [0, n_keep) to y, n_split + [0, n_keep) to y2
  int64_t n_keep = INT64_MAX;
};

struct Product {
  ProductKind kind = kProductLinear;
  int dtype = DTP_BF16;
  const void* a0 = nullptr;  // a1: the up projection, or the second segment's matrix
  const void* a1 = nullptr;
  const void* b = nullptr;
  int64_t lda = 0, ldb = 0;
  bool at = false, bt = false;  // element (row, k) at [k * ld + row] instead of [row * ld + k]
  int M = 0;
  int64_t N = 0, K = 0;  // K per segment
  int segments = 1;      // contraction over a0 and then, from column b_seg of B's rows on, over a1
  int64_t b_seg = 0;
  ProductOut out;
};

// ---- the products of an operator
inline int64_t pad32(int64_t n) { return (n + 31) / 32 * 32; }

inline Product forward_product(ProductKind kind, int64_t T, int K, int N, int dtype) {
  Product p;
  p.kind = kind;
  p.dtype = dtype;
  p.lda = p.ldb = K;
  p.M = N;
  p.N = T;
  p.K = K;
  return p;
}

// dx of n_parts stacked weight matrices: contraction over their rows.
inline Product dx_product(int64_t T, int K, int N, int parts, int ld, int dtype) {
  Product p;
  p.kind = kProductGrad;
  p.dtype = dtype;
  p.at = true;
  p.lda = K;
  p.ldb = (int64_t)parts * ld;
  p.M = K;
  p.N = T;
  p.K = N;
  p.segments = parts;
  p.b_seg = ld;
  return p;
}

inline Product dw_product(int64_t T, int K, int N, int parts, int ld, int dtype) {
  Product p;
  p.kind = kProductGrad;
  p.dtype = dtype;
  p.at = p.bt = true;
  p.lda = K;
  p.ldb = (int64_t)parts * ld;
  p.M = K;
  p.N = parts == 1 ? N : (int64_t)parts * ld;
  p.K = T;
  if (parts > 1) {
    p.out.n_split = ld;
    p.out.n_keep = N;
  }
  return p;
}

// Whether dz is formed on its own: with an activation, and where the bf16 kernels cannot take dy's
// rows in 16-byte pieces.
inline bool needs_pass(int N, int dtype, bool gated, bool with_act) {
  return gated || with_act || (dtype == DTP_BF16 && N % 8 != 0);
}

// ---- their launches, on a GPU of `cus` compute units
// Runs of a few-token product, and how many a block takes: the contraction is split where the
// features alone would leave half of the CUs idle and every wavefront keeps at least four runs.
inline void choose_stream(const Product& p, int cus, int64_t es, int& runs, int& per) {
  runs = (int)((p.K * es + 127) / 128);
  const int blocks = (p.M + 15) / 16;
  int splits = 1;
  while (blocks * splits < cus / 2 && runs / (splits * 2) >= 32) splits *= 2;
  per = (runs + splits - 1) / splits;
}

// -- bf16
struct ShapeBf16 {
  bool stream = false;
  int tile = 0;        // of kTilesBf16
  int splits = 1, per = 0, nq = 0;
};

// The tile and the splits of the contraction by the launch's estimated length in us: a CU's items, one
// stage of 64 columns after the other, half of the operands' bytes at memory speed (the other half is
// read beside the products), and the join of the parts.  The times per stage and item were fitted to
// launches of every tile and split.
struct Tile {
  int m, n;        // rows of A and of B
  int per_cu;      // blocks of a CU
  double alone, shared;  // us per stage: one item per CU, several
  double item;     // us per item beside its stages: results, the first copies
};
constexpr Tile kTilesBf16[] = {{256, 256, 1, 1.28, 1.32, 5.0}, {128, 128, 2, 0.50, 0.49, 1.0}, {128, 64, 3, 0.39, 0.33, 0.8}};

// Up to 8 tokens the weights are streamed into registers, and up to 16 where they are few: each block
// reads the tokens too, as many bytes as of weights at 16 tokens.  14,336 x 4,096, streamed and in tiles:
// 26.2 us and 27.1 for 8 tokens, 28.2 and 27.4 for 12, 31.4 and 28.0 for 16; 4,096 x 14,336: 31.7 and 27.5
// for 12; 4,096 x 4,096: 8.8 and 11.1 for 8, 10.0 and 11.4 for 16; a gated block of 4,096 x 14,336: 48.1
// and 48.7 for 8, 51.0 and 46.8 for 16.
inline bool streams_bf16(const Product& p) {
  if (p.at || p.bt) return false;
  return p.N <= 8 || (p.N <= kStreamTokens && (int64_t)p.M * p.K <= ((int64_t)1 << 24));
}

inline ShapeBf16 choose_bf16(const Product& p, int cus) {
  ShapeBf16 s;
  const bool gated = p.kind == kProductGated;
  if (streams_bf16(p)) {
    s.stream = true;
    choose_stream(p, cus, 2, s.nq, s.per);
    s.splits = (s.nq + s.per - 1) / s.per;
    return s;
  }
  // every item has an even number of stages
  s.nq = (int)((p.K + 2 * kRowStage - 1) / (2 * kRowStage)) * 2 * p.segments;
  const double M = (gated ? 2.0 : 1.0) * p.M, N = (double)p.N;
  const double stream = 2.0 * (M + N) * (double)p.K * p.segments / 5.5e6;  // us at 5.5 TB/s
  double best = 1e30;
  for (int i = 0; i < 3; ++i) {
    const Tile& t = kTilesBf16[i];
    const int64_t tiles = (((int64_t)M + t.m - 1) / t.m) * ((p.N + t.n - 1) / t.n);
    for (int splits = 1; splits <= std::min(32, s.nq / 2); ++splits) {
      const int per = (s.nq / 2 + splits - 1) / splits * 2;
      const int real = (s.nq + per - 1) / per;
      if (real != splits) continue;
      const int64_t items = (tiles * splits + cus - 1) / cus;  // of a CU
      double us = (double)items * (per * (items > 1 ? t.shared : t.alone) + t.item);
      us += 0.5 * stream;
      if (splits > 1) us += 3.0 + 8.0 * splits * M * N / 5e6;  // 32-bit parts written and read
      if (us < best) {
        best = us;
        s.tile = i;
        s.per = per;
        s.splits = splits;
      }
    }
  }
  return s;
}

// -- fp32
// us of a CU per stage and 64 x 64 sums in tiles of 128 and of 64, and of an item that has the CU to
// itself (in tiles of 128, whose four wavefronts leave the SIMDs one each).
constexpr double kBig = 0.0158 * kStageF32, kSmall = 0.0195 * kStageF32, kBigAlone = 0.0190 * kStageF32, kSmallAlone = 0.0260 * kStageF32;

// Tiles of one launch: a launch takes fewer than 2^32 threads, and a tile has at most 512.  More
// tiles are more launches.
constexpr int64_t kMostTilesF32 = (int64_t)1 << 22;

struct ShapeF32 {
  bool stream = false;
  int f = 2, splits = 1, per = 0, stages = 0, m_tiles = 0;
  int64_t n_tiles = 0;
  int threads() const { return f == 2 ? 256 : 512; }
  // Tiles of the launch that starts with tile `first`.
  int64_t launch_tiles(int64_t first) const { return std::min(m_tiles * n_tiles - first, kMostTilesF32); }
};

inline ShapeF32 choose_f32(const Product& p, int cus) {
  ShapeF32 s;
  const bool gated = p.kind == kProductGated;
  if (!p.at && !p.bt && p.N <= kStreamTokens) {
    s.stream = true;
    choose_stream(p, cus, 4, s.stages, s.per);
    s.splits = (s.stages + s.per - 1) / s.per;
    return s;
  }
  s.stages = (int)((p.K + kStageF32 - 1) / kStageF32);
  const int nq = s.stages * p.segments;
  const double planes = gated ? 2.0 : 1.0;
  double best = 1e30;
  for (int f = 1; f <= 2; ++f) {
    const int rows = gated ? 64 : 64 * f;
    const int64_t m_tiles = (p.M + rows - 1) / rows, n_tiles = (p.N + 64 * f - 1) / (64 * f);
    const double sums = (gated ? 2.0 : f) * f;  // 64 x 64 of them in a tile
    for (int splits = 1; splits <= std::min(32, std::max(1, nq / 2)); ++splits) {
      const int per = (nq + splits - 1) / splits;
      if ((nq + per - 1) / per != splits) continue;
      const int64_t items = (m_tiles * n_tiles * splits + cus - 1) / cus;  // of a CU
      const double rate = items > 1 ? (f == 2 ? kBig : kSmall) : (f == 2 ? kBigAlone : kSmallAlone);
      double us = (double)items * (per * sums * rate + 1.0);
      if (splits > 1) us += 3.0 + 8.0 * splits * planes * p.M * (double)p.N / 5e6;  // parts written and read
      if (us < best) {
        best = us;
        s.f = f;
        s.m_tiles = (int)m_tiles;
        s.n_tiles = n_tiles;
        s.per = per;
        s.splits = splits;
      }
    }
  }
  return s;
}

}  // namespace dtp
