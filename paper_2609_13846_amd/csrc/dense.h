// The products of a dense decoder layer (linear and gated operators): their launches, and the
// activations and result writes that their kernels share (gfx950).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dense_plan.h"
#include "dtp_internal.h"
#include "tile_mfma.h"

namespace dtp {

// ---- arguments of the dense operators (dense.hip)
struct Range {  // a buffer of the caller's
  const void* p;
  size_t bytes;
  const char* name;
  int align = 16;
  int in_place = -1;  // the one input, by its place in the list, that an output may be in place of
};
// Alignment, memory and room of the buffers that are not NULL.
dtp_status check_ranges(const Range* r, int n);
// No output overlaps an input (but in place where `in_place` says so) or another output.
dtp_status check_disjoint(const Range* outs, int n_outs, const Range* ins, int n_ins);

// A call's scratch: the caller's workspace, or stream-ordered memory that is returned with it.
struct Workspace {
  char* base = nullptr;
  char* owned = nullptr;
  hipStream_t s = nullptr;
  Workspace() = default;
  Workspace(const Workspace&) = delete;
  Workspace& operator=(const Workspace&) = delete;
  ~Workspace();
  dtp_status open(void* given, int64_t given_bytes, int64_t need, hipStream_t stream);
};

// Enqueues the product; workspace of product_bytes(p) bytes, 256-byte pieces.
size_t product_bytes(const Product& p);
dtp_status launch_product(const Product& p, char* workspace, hipStream_t s);
size_t product_bytes_bf16(const Product& p);  // dense_bf16.hip
dtp_status launch_product_bf16(const Product& p, char* workspace, hipStream_t s);
size_t product_bytes_f32(const Product& p);  // dense_f32.hip
dtp_status launch_product_f32(const Product& p, char* workspace, hipStream_t s);

#ifdef __HIPCC__

// One element type's storage and its conversions.  kWide: elements of 16 bytes.
template <typename S>
struct Elem;
template <>
struct Elem<uint16_t> {
  static constexpr int kWide = 8;
  __device__ static __forceinline__ float load(uint16_t v) { return bf16_to_f32(v); }
  __device__ static __forceinline__ uint16_t store(float v) { return f32_to_bf16(v); }
};
template <>
struct Elem<float> {
  static constexpr int kWide = 4;
  __device__ static __forceinline__ float load(float v) { return v; }
  __device__ static __forceinline__ float store(float v) { return v; }
};

// sigma(w) and 1 - sigma(w), each without cancellation.  bf16 results take the hardware's
// exponential and reciprocal: the smaller of the two is off by about (|w| + 2) 2^-23 of itself (the
// product of w and log2 e is rounded), less than 2^-16 up to where the exponential underflows
// (|w| = 87); a result is rounded to within 2^-9.
template <typename S>
__device__ __forceinline__ void sigmoid(float w, float& s, float& rest) {
  const bool fast = sizeof(S) == 2;
  const float e = fast ? __expf(-fabsf(w)) : expf(-fabsf(w));
  const float big = fast ? __builtin_amdgcn_rcpf(1.0f + e) : 1.0f / (1.0f + e);
  const float small = e * big;
  s = w < 0.0f ? small : big;
  rest = w < 0.0f ? big : small;
}

constexpr float kGelu = 0.7978845608028654f, kGelu3 = 0.044715f;  // sqrt(2 / pi)

// 1 + tanh(w) = 2 sigma(2 w), so gelu(z) = z sigma(2 w), w = sqrt(2 / pi) (z + 0.044715 z^3).
template <typename S>
__device__ __forceinline__ float activate(int act, float z) {
  if (act == DTP_ACT_NONE) return z;
  float s, rest;
  sigmoid<S>(act == DTP_ACT_SILU ? z : 2.0f * kGelu * (z + kGelu3 * z * z * z), s, rest);
  return z * s;
}

// act(z) and act'(z) = sigma + z sigma (1 - sigma) w'.  Beyond |z| = 30 the second term of
// gelu' is nothing, where z^2 may be infinite.
template <typename S>
__device__ __forceinline__ void activate_grad(int act, float z, float& a, float& da) {
  if (act == DTP_ACT_NONE) {
    a = z;
    da = 1.0f;
    return;
  }
  float s, rest;
  if (act == DTP_ACT_SILU) {
    sigmoid<S>(z, s, rest);
    da = s * (1.0f + z * rest);
  } else {
    const float c = z > 30.0f ? 30.0f : (z < -30.0f ? -30.0f : z);  // NaN stays
    sigmoid<S>(2.0f * kGelu * (c + kGelu3 * c * c * c), s, rest);
    da = s + c * s * rest * 2.0f * kGelu * (1.0f + 3.0f * kGelu3 * c * c);
  }
  a = z * s;
}

// 16 bytes at any address of the element type's alignment: global memory takes such loads and stores
// whole, so that rows of odd lengths need no path of their own.
typedef u32x4 __attribute__((aligned(2))) u32x4_any;
typedef f32x4 __attribute__((aligned(4))) f32x4_any;

// W elements of a row, or the `count` that are left of it.
template <typename S, int W>
__device__ __forceinline__ void load_row(const S* p, int count, float (&v)[W]) {
  if (count >= W) {
    union {
      u32x4 q[W * sizeof(S) / 16];
      S e[W];
    } u;
#pragma unroll
    for (int i = 0; i < (int)(W * sizeof(S) / 16); ++i) u.q[i] = reinterpret_cast<const u32x4_any*>(p)[i];
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = Elem<S>::load(u.e[i]);
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = i < count ? Elem<S>::load(p[i]) : 0.0f;
  }
}

template <typename S, int W>
__device__ __forceinline__ void store_row(S* p, int count, const float (&v)[W]) {
  if (count >= W) {
    union {
      u32x4 q[W * sizeof(S) / 16];
      uint32_t d[W * sizeof(S) / 4];
      float f[W * sizeof(S) / 4];
    } u;
    if constexpr (sizeof(S) == 2) {
#pragma unroll
      for (int i = 0; i < W / 2; ++i) u.d[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < W; ++i) u.f[i] = v[i];
    }
#pragma unroll
    for (int i = 0; i < (int)(W * sizeof(S) / 16); ++i) reinterpret_cast<u32x4_any*>(p)[i] = u.q[i];
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i)
      if (i < count) p[i] = Elem<S>::store(v[i]);
  }
}

// Writes W (8 for bf16, 4 for fp32) results from (n, m) on, m a multiple of W.  c0: the sums;
// c1: the up projection's.  The result is rounded once, here.
template <typename S, ProductKind KIND, int W>
__device__ __forceinline__ void write_product(const ProductOut& o, int64_t n, int m, int M, const float (&c0)[W],
                                              const float (&c1)[W]) {
  const int count = M - m;
  if (count <= 0) return;
  float v[W];
  if constexpr (KIND == kProductLinear) {
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = c0[i];
    if (o.bias) {
      float b[W];
      load_row((const S*)o.bias + m, count, b);
#pragma unroll
      for (int i = 0; i < W; ++i) v[i] += b[i];
    }
    if (o.pre) store_row(o.pre + n * M + m, count, v);
    if (o.act != DTP_ACT_NONE) {
#pragma unroll
      for (int i = 0; i < W; ++i) v[i] = activate<S>(o.act, v[i]);
    }
    if (o.residual) {
      float r[W];
      load_row((const S*)o.residual + n * M + m, count, r);
#pragma unroll
      for (int i = 0; i < W; ++i) v[i] = fmaf(o.alpha, v[i], r[i]);
    } else {
#pragma unroll
      for (int i = 0; i < W; ++i) v[i] *= o.alpha;
    }
    store_row((S*)o.y + n * M + m, count, v);
  } else if constexpr (KIND == kProductGated) {
    if (o.pre) {
      store_row(o.pre + 2 * n * M + m, count, c0);
      store_row(o.pre + (2 * n + 1) * M + m, count, c1);
    }
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = activate<S>(o.act, c0[i]) * c1[i];
    store_row((S*)o.y + n * M + m, count, v);
  } else {
    const bool second = n >= o.n_split;
    const int64_t row = second ? n - o.n_split : n;
    if (row >= o.n_keep) return;
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = o.alpha * c0[i];
    S *const y1 = (S*)o.y, *const y2 = (S*)o.y2;
    store_row((second ? y2 : y1) + row * M + m, count, v);
  }
}

#endif  // __HIPCC__

}  // namespace dtp
