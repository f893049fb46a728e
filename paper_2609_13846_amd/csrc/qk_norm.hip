// Per-head RMS norms of queries and keys with the rotation by position (dtp_qk_norm_rotate_*).
//
//   n = gamma v / r, r = sqrt(mean v^2 + eps);  out = R(a) n, R the rotation of the column pairs.
// Backward, with dn = R(-a) dout (a rotation's transpose) and dhat = gamma dn:
//   dgamma = sum dn v / r,   dv = (dhat - (v / r) mean(dhat v / r)) / r.
//
// A head's columns are taken as dh / 2 pairs: (j, j + R/2) for the rotated ones, and the rest of
// the head split in the middle the same way, so that both columns of a pair are in one lane and the
// rotation needs no exchange.  A lane holds V pairs in two V-wide pieces, a power of two of lanes
// a head (the norm's sum is a few exchanges among them), and a wavefront several heads of a
// token at a time.  Squares are summed in 32 bits, and again in 64 for a head where they leave that
// range, so that a norm does not depend on a head's scale.  A token's angles are formed once per wavefront, one pair per lane, in 64 bits
// (position * inv_freq in turns, of which only the fraction matters), and shared through LDS.
//
// Bound by memory: 32,768 tokens of 24 heads of 128 in bf16 take 83 us forward (0.40 GB, 4.9 TB/s; a
// copy 4.7) and 148 backward (0.60 GB, 4.1 TB/s), and 8 for the join of dgamma.
#include <algorithm>
#include <cmath>

#include "dense.h"

namespace dtp {
namespace {

constexpr int kMaxHeadDim = 256;
constexpr int kMaxPairs = kMaxHeadDim / 2;

struct QkArgs {
  const void *q, *k, *gamma_q, *gamma_k, *dq_out, *dk_out;
  void *q_out, *k_out;  // dq, dk of the backward pass
  int64_t q_stride, k_stride;
  const int32_t* positions;
  const float* inv_freq;
  float* partial;  // backward: [blocks][2][dh]
  float eps;
  int64_t T;
  int H, G, dh, half;   // half: rotated pairs, R / 2
  int lanes;            // of a head, a power of two
  int slices;           // wavefronts that share a token's heads
};

// Cosine and sine of a_j for the token's pairs, one lane each.
__device__ __forceinline__ void angles(const QkArgs& p, int64_t t, int lane, float2* cs) {
  const double pos = (double)p.positions[t];
  for (int j = lane; j < p.half; j += 64) {
    const double turns = pos * (double)p.inv_freq[j] * 0.15915494309189533577;  // 1 / (2 pi)
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    cs[j] = make_float2(c, s);
  }
}

// Column of pair j's first element; its second is half (rotated) or rest / 2 columns further.
__device__ __forceinline__ int pair_column(const QkArgs& p, int j) { return j < p.half ? j : j + p.half; }
__device__ __forceinline__ int pair_reach(const QkArgs& p, int j) { return j < p.half ? p.half : p.dh / 2 - p.half; }

template <typename S, int V>
__device__ __forceinline__ void load_piece(const S* p, float (&v)[V]) {
  struct alignas(V * sizeof(S)) Piece {
    S e[V];
  };
  const Piece x = *reinterpret_cast<const Piece*>(p);
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = Elem<S>::load(x.e[i]);
}

template <typename S, int V>
__device__ __forceinline__ void store_piece(S* p, const float (&v)[V]) {
  struct alignas(V * sizeof(S)) Piece {
    S e[V];
  };
  Piece x;
#pragma unroll
  for (int i = 0; i < V; ++i) x.e[i] = Elem<S>::store(v[i]);
  *reinterpret_cast<Piece*>(p) = x;
}

template <typename F>
__device__ __forceinline__ F head_sum(F v, int lanes) {
  for (int d = 1; d < lanes; d *= 2) v += __shfl_xor(v, d);
  return v;
}

// NS pieces of V pairs per lane.  A block: four wavefronts, each walking (token, slice) items.
template <typename S, int V, int NS, bool BACKWARD>
__global__ void __launch_bounds__(256) qk_kernel(QkArgs p) {
  __shared__ float2 cs[4][kMaxPairs];
  __shared__ float sums[4][2][kMaxHeadDim];
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const int per = 64 / p.lanes, head_lane = lane % p.lanes, slot = lane / p.lanes;
  const int q_rounds = (p.H + per - 1) / per, rounds = q_rounds + (p.G + per - 1) / per;
  const bool norm = p.gamma_q != nullptr;
  float dg[2][NS][2][V] = {};  // dgamma of this lane's columns: queries, keys
  for (int64_t item = (int64_t)blockIdx.x * 4 + wave; item < p.T * p.slices; item += (int64_t)gridDim.x * 4) {
    const int64_t t = item / p.slices;
    const int slice = (int)(item - t * p.slices);
    if (p.half > 0) {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the reads of the item before are done
      angles(p, t, lane, cs[wave]);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    for (int r = slice; r < rounds; r += p.slices) {
      const bool is_q = r < q_rounds;
      const int head = (is_q ? r : r - q_rounds) * per + slot, heads = is_q ? p.H : p.G;
      const bool in = head < heads;
      const S* src = (const S*)(is_q ? p.q : p.k) + t * (is_q ? p.q_stride : p.k_stride) + (int64_t)head * p.dh;
      const int64_t dense = (t * heads + head) * p.dh;
      const S* gamma = (const S*)(is_q ? p.gamma_q : p.gamma_k);
      float v[NS][2][V] = {}, g[NS][2][V] = {};
      bool on[NS];
      int c0[NS], c1[NS], pair[NS];
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        pair[s] = (head_lane + s * p.lanes) * V;
        on[s] = in && pair[s] < p.dh / 2;
        c0[s] = pair_column(p, pair[s]);
        c1[s] = c0[s] + pair_reach(p, pair[s]);
        if (on[s]) {
          load_piece<S, V>(src + c0[s], v[s][0]);
          load_piece<S, V>(src + c1[s], v[s][1]);
          if (norm) {
            load_piece<S, V>(gamma + c0[s], g[s][0]);
            load_piece<S, V>(gamma + c1[s], g[s][1]);
          }
        }
      }
      float inv = 1.0f;
      if (norm) {
        float sq = 0.0f;
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
          for (int i = 0; i < V; ++i) sq = fmaf(v[s][0][i], v[s][0][i], fmaf(v[s][1][i], v[s][1][i], sq));
        const float r2 = head_sum(sq, p.lanes) / (float)p.dh + p.eps;
        if (r2 > 0x1p-100f && r2 < INFINITY) {
          inv = 1.0f / sqrtf(r2);
        } else {  // squares outside the range of 32 bits (or zeros, or not finite); all of a head's lanes
          double wide = 0.0;
#pragma unroll
          for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int i = 0; i < V; ++i) wide += (double)v[s][0][i] * v[s][0][i] + (double)v[s][1][i] * v[s][1][i];
          wide = fma((double)p.dh, (double)p.eps, head_sum(wide, p.lanes));
          const int e = __builtin_amdgcn_frexp_exp(wide) & ~1;
          inv = ldexpf(1.0f / sqrtf((float)ldexp(wide, -e) / (float)p.dh), -e / 2);
        }
        if (!in) inv = 0.0f;  // no head: nothing for dgamma, whatever eps
      }
      if constexpr (!BACKWARD) {
        S* out = (S*)(is_q ? p.q_out : p.k_out) + dense;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          float a[V], b[V];
#pragma unroll
          for (int i = 0; i < V; ++i) {
            a[i] = norm ? g[s][0][i] * (v[s][0][i] * inv) : v[s][0][i];
            b[i] = norm ? g[s][1][i] * (v[s][1][i] * inv) : v[s][1][i];
            if (pair[s] < p.half) {
              const float2 w = cs[wave][pair[s] + i];
              const float x = a[i], y = b[i];
              a[i] = x * w.x - y * w.y;
              b[i] = y * w.x + x * w.y;
            }
          }
          if (on[s]) {
            store_piece<S, V>(out + c0[s], a);
            store_piece<S, V>(out + c1[s], b);
          }
        }
      } else {
        const S* dout = (const S*)(is_q ? p.dq_out : p.dk_out) + dense;
        S* out = (S*)(is_q ? p.q_out : p.k_out) + dense;
        float d[NS][2][V] = {};
        float dot = 0.0f;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          if (on[s]) {
            load_piece<S, V>(dout + c0[s], d[s][0]);
            load_piece<S, V>(dout + c1[s], d[s][1]);
          }
#pragma unroll
          for (int i = 0; i < V; ++i) {
            if (pair[s] < p.half) {
              const float2 w = cs[wave][pair[s] + i];
              const float x = d[s][0][i], y = d[s][1][i];
              d[s][0][i] = x * w.x + y * w.y;
              d[s][1][i] = y * w.x - x * w.y;
            }
            if (norm) {
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float hat = v[s][e][i] * inv;
                if (is_q)
                  dg[0][s][e][i] = fmaf(d[s][e][i], hat, dg[0][s][e][i]);
                else
                  dg[1][s][e][i] = fmaf(d[s][e][i], hat, dg[1][s][e][i]);
                d[s][e][i] *= g[s][e][i];
                v[s][e][i] = hat;
                dot = fmaf(d[s][e][i], hat, dot);
              }
            }
          }
        }
        if (norm) {
          const float mean = head_sum(dot, p.lanes) / (float)p.dh;
#pragma unroll
          for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
              for (int i = 0; i < V; ++i) d[s][e][i] = inv * (d[s][e][i] - v[s][e][i] * mean);
        }
#pragma unroll
        for (int s = 0; s < NS; ++s)
          if (on[s]) {
            store_piece<S, V>(out + c0[s], d[s][0]);
            store_piece<S, V>(out + c1[s], d[s][1]);
          }
      }
    }
  }
  if constexpr (BACKWARD) {
    if (p.partial == nullptr) return;
    // over the wavefront's heads, then the block's wavefronts, in a fixed order
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
      for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            float x = dg[w][s][e][i];
            for (int d = p.lanes; d < 64; d *= 2) x += __shfl_xor(x, d);
            const int pair = (head_lane + s * p.lanes) * V;
            if (slot == 0 && pair < p.dh / 2)
              sums[wave][w][pair_column(p, pair) + (e ? pair_reach(p, pair) : 0) + i] = x;
          }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * p.dh; c += 256) {
      const int w = c / p.dh, i = c % p.dh;
      p.partial[(int64_t)blockIdx.x * 2 * p.dh + c] = (sums[0][w][i] + sums[1][w][i]) + (sums[2][w][i] + sums[3][w][i]);
    }
  }
}

// dgamma from the blocks' partial sums; a block per column of q's, then k's.
template <typename S>
__global__ void __launch_bounds__(64)
join_gamma_kernel(const float* __restrict__ partial, int blocks, int dh, S* __restrict__ dgamma_q, S* __restrict__ dgamma_k) {
  const int c = blockIdx.x;
  double v = 0.0;
  for (int b = threadIdx.x; b < blocks; b += 64) v += (double)partial[(int64_t)b * 2 * dh + c];
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  if (threadIdx.x == 0) (c < dh ? dgamma_q : dgamma_k)[c % dh] = Elem<S>::store((float)v);
}

template <typename S>
__global__ void zero_gamma_kernel(int dh, S* dgamma_q, S* dgamma_k) {
  for (int i = threadIdx.x; i < dh; i += 256) dgamma_q[i] = dgamma_k[i] = S(0);
}

constexpr int kBackwardBlocks = 1024;

int64_t backward_blocks(int64_t T) { return std::min<int64_t>((T + 3) / 4, kBackwardBlocks); }

dtp_status check_qk_sizes(int64_t T, int H, int G, int dh, int dtype) {
  DTP_CHECK(T >= 0, DTP_ERR_INVALID_ARG, "n_tokens=%lld is negative", (long long)T);
  DTP_CHECK(H > 0 && G > 0 && dh > 0, DTP_ERR_INVALID_ARG, "every size must be positive (H=%d G=%d dh=%d)", H, G, dh);
  DTP_CHECK(H % G == 0, DTP_ERR_INVALID_ARG, "H=%d is not a multiple of G=%d", H, G);
  DTP_CHECK(dh % 2 == 0, DTP_ERR_INVALID_ARG, "head_dim=%d is odd", dh);
  DTP_CHECK(dh <= kMaxHeadDim && H <= 65536 && T <= ((int64_t)1 << 30), DTP_ERR_UNSUPPORTED,
            "shape too large (head_dim <= %d, heads <= 65536, tokens <= 2^30)", kMaxHeadDim);
  DTP_CHECK(dtype == DTP_BF16 || dtype == DTP_F32, DTP_ERR_UNSUPPORTED, "dtype %d", dtype);
  return DTP_OK;
}

template <typename S, bool BACKWARD>
void launch_qk(QkArgs p, int64_t blocks, int V, hipStream_t s) {
  auto run = [&](auto v, auto ns) {
    qk_kernel<S, decltype(v)::value, decltype(ns)::value, BACKWARD><<<(unsigned)blocks, 256, 0, s>>>(p);
  };
  using std::integral_constant;
  if (V == 8)
    run(integral_constant<int, 8>(), integral_constant<int, 1>());
  else if (V == 4)
    run(integral_constant<int, 4>(), integral_constant<int, 1>());
  else if (V == 2)
    run(integral_constant<int, 2>(), integral_constant<int, 1>());
  else
    run(integral_constant<int, 1>(), integral_constant<int, 2>());
}

// The arguments that both passes share, checked; V: pairs per piece.
dtp_status prepare(QkArgs& p, int& V, int64_t T, int H, int G, int dh, int dtype, const void* q, int64_t q_stride,
                   const void* k, int64_t k_stride, const void* gamma_q, const void* gamma_k, float eps,
                   const int32_t* positions, const float* inv_freq, int rot) {
  dtp_status st = check_qk_sizes(T, H, G, dh, dtype);
  if (st != DTP_OK) return st;
  DTP_CHECK((gamma_q == nullptr) == (gamma_k == nullptr), DTP_ERR_INVALID_ARG,
            "gamma_q and gamma_k must be given together");
  DTP_CHECK((positions == nullptr) == (inv_freq == nullptr) && (positions == nullptr) == (rot == 0),
            DTP_ERR_INVALID_ARG, "positions, inv_freq and rot_dim must be given together");
  DTP_CHECK(rot >= 0 && rot <= dh && rot % 2 == 0, DTP_ERR_INVALID_ARG, "rot_dim=%d is odd or outside [0, %d]", rot, dh);
  DTP_CHECK(gamma_q || positions, DTP_ERR_INVALID_ARG, "neither a norm nor a rotation");
  DTP_CHECK(std::isfinite(eps) && eps >= 0.0f, DTP_ERR_INVALID_ARG, "eps=%g must be finite and >= 0", (double)eps);
  DTP_CHECK(q_stride >= (int64_t)H * dh && k_stride >= (int64_t)G * dh, DTP_ERR_INVALID_ARG,
            "a token's heads overlap the next token's (strides %lld, %lld)", (long long)q_stride, (long long)k_stride);
  DTP_CHECK(q_stride <= ((int64_t)1 << 32) && k_stride <= ((int64_t)1 << 32), DTP_ERR_UNSUPPORTED, "strides beyond 2^32");
  DTP_CHECK(T == 0 || (q && k), DTP_ERR_INVALID_ARG, "q or k is NULL");
  p = QkArgs{};
  p.q = q;
  p.k = k;
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.gamma_q = gamma_q;
  p.gamma_k = gamma_k;
  p.eps = eps;
  p.positions = positions;
  p.inv_freq = inv_freq;
  p.T = T;
  p.H = H;
  p.G = G;
  p.dh = dh;
  p.half = rot / 2;
  // The widest pieces, at most 16 bytes, in which every pair's two columns are whole and aligned.
  const int es = dtype == DTP_BF16 ? 2 : 4;
  const int64_t all = (int64_t)(rot / 2) | (dh / 2 - rot / 2) | dh | q_stride | k_stride;
  const uintptr_t at = (uintptr_t)q | (uintptr_t)k;
  V = 16 / es;
  while (V > 1 && (all % V != 0 || at % (uintptr_t)(V * es) != 0)) V /= 2;
  p.lanes = 1;
  while (p.lanes * V * (V == 1 ? 2 : 1) < dh / 2) p.lanes *= 2;
  return DTP_OK;
}

size_t qk_bytes(int64_t T, int64_t stride, int64_t heads, int dh, size_t es) {
  return T == 0 ? 0 : es * (size_t)((T - 1) * stride + heads * dh);
}

}  // namespace
}  // namespace dtp

using namespace dtp;

extern "C" {

int64_t dtp_qk_norm_rotate_workspace(int64_t n_tokens, int32_t n_q_heads, int32_t n_kv_groups, int32_t head_dim,
                                     dtp_dtype dtype) {
  int64_t n = -1;
  (void)guarded([&]() -> dtp_status {
    clear_error();
    const dtp_status st = check_qk_sizes(n_tokens, n_q_heads, n_kv_groups, head_dim, dtype);
    if (st == DTP_OK) n = (int64_t)sizeof(float) * backward_blocks(n_tokens) * 2 * head_dim;
    return st;
  });
  return n;
}

dtp_status dtp_qk_norm_rotate_forward(int64_t n_tokens, int32_t n_q_heads, int32_t n_kv_groups, int32_t head_dim,
                                      dtp_dtype dtype, const void* q, int64_t q_stride, const void* k,
                                      int64_t k_stride, const void* gamma_q, const void* gamma_k, float eps,
                                      const int32_t* positions, const float* inv_freq, int32_t rot_dim, void* q_out,
                                      void* k_out, void* stream) {
  return guarded([&]() -> dtp_status {
    clear_error();
    const int64_t T = n_tokens;
    const int H = n_q_heads, G = n_kv_groups, dh = head_dim;
    QkArgs p;
    int V;
    dtp_status st = prepare(p, V, T, H, G, dh, dtype, q, q_stride, k, k_stride, gamma_q, gamma_k, eps, positions,
                            inv_freq, rot_dim);
    if (st != DTP_OK || T == 0) return st;
    DTP_CHECK(q_out && k_out, DTP_ERR_INVALID_ARG, "q_out or k_out is NULL");
    const int es = dtype == DTP_BF16 ? 2 : 4;
    const size_t nq = (size_t)es * T * H * dh, nk = (size_t)es * T * G * dh;
    const Range in[] = {{q, qk_bytes(T, q_stride, H, dh, es), "q", es}, {k, qk_bytes(T, k_stride, G, dh, es), "k", es},
                        {gamma_q, (size_t)es * dh, "gamma_q"}, {gamma_k, (size_t)es * dh, "gamma_k"},
                        {positions, sizeof(int32_t) * (size_t)T, "positions"},
                        {inv_freq, sizeof(float) * (size_t)(rot_dim / 2), "inv_freq"}};
    const Range out[] = {{q_out, nq, "q_out", 16, q_stride == (int64_t)H * dh ? 0 : -1},
                         {k_out, nk, "k_out", 16, k_stride == (int64_t)G * dh ? 1 : -1}};
    if ((st = check_disjoint(out, 2, in, 6)) != DTP_OK || (st = check_ranges(in, 6)) != DTP_OK ||
        (st = check_ranges(out, 2)) != DTP_OK)
      return st;
    p.q_out = q_out;
    p.k_out = k_out;
    const int per = 64 / p.lanes, rounds = (H + per - 1) / per + (G + per - 1) / per;
    // Few tokens: several wavefronts share a token's heads, while there are compute units for them.
    p.slices = (int)std::max<int64_t>(1, std::min<int64_t>(rounds, 4096 / std::max<int64_t>(T, 1)));
    const int64_t blocks = std::min<int64_t>((T * p.slices + 3) / 4, (int64_t)1 << 20);
    if (dtype == DTP_BF16)
      launch_qk<uint16_t, false>(p, blocks, V, (hipStream_t)stream);
    else
      launch_qk<float, false>(p, blocks, V, (hipStream_t)stream);
    DTP_HIP(hipGetLastError());
    return DTP_OK;
  });
}

dtp_status dtp_qk_norm_rotate_backward(int64_t n_tokens, int32_t n_q_heads, int32_t n_kv_groups, int32_t head_dim,
                                       dtp_dtype dtype, const void* q, int64_t q_stride, const void* k,
                                       int64_t k_stride, const void* gamma_q, const void* gamma_k, float eps,
                                       const int32_t* positions, const float* inv_freq, int32_t rot_dim,
                                       const void* dq_out, const void* dk_out, void* dq, void* dk, void* dgamma_q,
                                       void* dgamma_k, void* workspace, int64_t workspace_bytes, void* stream) {
  return guarded([&]() -> dtp_status {
    clear_error();
    const int64_t T = n_tokens;
    const int H = n_q_heads, G = n_kv_groups, dh = head_dim;
    hipStream_t s = (hipStream_t)stream;
    QkArgs p;
    int V;
    dtp_status st = prepare(p, V, T, H, G, dh, dtype, q, q_stride, k, k_stride, gamma_q, gamma_k, eps, positions,
                            inv_freq, rot_dim);
    if (st != DTP_OK) return st;
    DTP_CHECK((dgamma_q == nullptr) == (dgamma_k == nullptr), DTP_ERR_INVALID_ARG,
              "dgamma_q and dgamma_k must be given together");
    DTP_CHECK(dgamma_q == nullptr || gamma_q, DTP_ERR_INVALID_ARG, "dgamma without a norm");
    DTP_CHECK(T == 0 || (dq_out && dk_out && dq && dk), DTP_ERR_INVALID_ARG, "dq_out, dk_out, dq or dk is NULL");
    const int es = dtype == DTP_BF16 ? 2 : 4;
    const size_t nq = (size_t)es * T * H * dh, nk = (size_t)es * T * G * dh;
    auto some = [T](const void* x) { return T ? x : nullptr; };
    const Range in[] = {{some(q), qk_bytes(T, q_stride, H, dh, es), "q", es},
                        {some(k), qk_bytes(T, k_stride, G, dh, es), "k", es},
                        {some(gamma_q), (size_t)es * dh, "gamma_q"}, {some(gamma_k), (size_t)es * dh, "gamma_k"},
                        {some(positions), sizeof(int32_t) * (size_t)T, "positions"},
                        {some(inv_freq), sizeof(float) * (size_t)(rot_dim / 2), "inv_freq"},
                        {some(dq_out), nq, "dq_out"}, {some(dk_out), nk, "dk_out"}};
    const Range out[] = {{some(dq), nq, "dq", 16, 6}, {some(dk), nk, "dk", 16, 7},
                         {dgamma_q, (size_t)es * dh, "dgamma_q"}, {dgamma_k, (size_t)es * dh, "dgamma_k"},
                         {workspace, (size_t)std::max<int64_t>(workspace_bytes, 0), "workspace"}};
    if ((st = check_disjoint(out, 5, in, 8)) != DTP_OK || (st = check_ranges(in, 8)) != DTP_OK ||
        (st = check_ranges(out, 4)) != DTP_OK)
      return st;
    if (T == 0) {
      if (dgamma_q == nullptr) return DTP_OK;
      if (dtype == DTP_BF16)
        zero_gamma_kernel<<<1, 256, 0, s>>>(dh, (uint16_t*)dgamma_q, (uint16_t*)dgamma_k);
      else
        zero_gamma_kernel<<<1, 256, 0, s>>>(dh, (float*)dgamma_q, (float*)dgamma_k);
      DTP_HIP(hipGetLastError());
      return DTP_OK;
    }
    const int64_t blocks = backward_blocks(T);
    Workspace ws;
    if ((st = ws.open(workspace, workspace_bytes, dgamma_q ? (int64_t)sizeof(float) * blocks * 2 * dh : 0, s)) != DTP_OK)
      return st;
    p.dq_out = dq_out;
    p.dk_out = dk_out;
    p.q_out = dq;
    p.k_out = dk;
    p.partial = dgamma_q ? (float*)ws.base : nullptr;
    p.slices = 1;
    if (dtype == DTP_BF16)
      launch_qk<uint16_t, true>(p, blocks, V, s);
    else
      launch_qk<float, true>(p, blocks, V, s);
    DTP_HIP(hipGetLastError());
    if (dgamma_q) {
      if (dtype == DTP_BF16)
        join_gamma_kernel<<<2 * dh, 64, 0, s>>>((const float*)ws.base, (int)blocks, dh, (uint16_t*)dgamma_q,
                                                (uint16_t*)dgamma_k);
      else
        join_gamma_kernel<<<2 * dh, 64, 0, s>>>((const float*)ws.base, (int)blocks, dh, (float*)dgamma_q,
                                                (float*)dgamma_k);
      DTP_HIP(hipGetLastError());
    }
    return DTP_OK;
  });
}

}  // extern "C"
