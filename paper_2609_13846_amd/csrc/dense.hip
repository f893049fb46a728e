// Entry points of the dense layer's products (dtp_linear_*, dtp_gated_*): argument checks, the
// plan of each call (its products and its workspace), and the passes beside the products:
//   activation_grad_kernel  dz from dy and the kept pre-activations
//   column_sums_kernel, join_sums_kernel  the bias's gradient
#include <algorithm>
#include <cmath>

#include "dense.h"

namespace dtp {

dtp_status check_disjoint(const Range* outs, int n_outs, const Range* ins, int n_ins) {
  auto overlap = [](const Range& a, const Range& b) {
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return a.p && b.p && a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
  };
  for (int i = 0; i < n_outs; ++i) {
    for (int j = 0; j < n_ins; ++j)
      DTP_CHECK(!overlap(outs[i], ins[j]) || (outs[i].in_place == j && outs[i].p == ins[j].p),
                DTP_ERR_INVALID_ARG, "%s overlaps %s", outs[i].name, ins[j].name);
    for (int j = i + 1; j < n_outs; ++j)
      DTP_CHECK(!overlap(outs[i], outs[j]), DTP_ERR_INVALID_ARG, "%s overlaps %s", outs[i].name, outs[j].name);
  }
  return DTP_OK;
}

dtp_status check_ranges(const Range* r, int n) {
  for (int i = 0; i < n; ++i) {
    if (r[i].p == nullptr) continue;
    DTP_CHECK(((uintptr_t)r[i].p & (r[i].align - 1)) == 0, DTP_ERR_INVALID_ARG, "%s must be %d-byte aligned",
              r[i].name, r[i].align);
    const dtp_status st = check_dev_buffer(r[i].p, r[i].bytes, r[i].name);
    if (st != DTP_OK) return st;
  }
  return DTP_OK;
}

dtp_status Workspace::open(void* given, int64_t given_bytes, int64_t need, hipStream_t stream) {
  s = stream;
  if (given != nullptr) {
    DTP_CHECK(given_bytes >= need, DTP_ERR_INVALID_ARG, "workspace has %lld bytes, the call needs %lld",
              (long long)given_bytes, (long long)need);
    const Range r{given, (size_t)given_bytes, "workspace"};
    base = (char*)given;
    return check_ranges(&r, 1);
  }
  if (need == 0) return DTP_OK;
  hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
  DTP_HIP(hipStreamIsCapturing(s, &st));
  DTP_CHECK(st == hipStreamCaptureStatusNone, DTP_ERR_UNSUPPORTED,
            "a call that is captured into a graph needs a workspace of %lld bytes", (long long)need);
  const hipError_t e = stream_alloc((void**)&owned, (size_t)need, s);
  if (e != hipSuccess) owned = nullptr, (void)hipGetLastError();
  DTP_CHECK(e == hipSuccess, e == hipErrorOutOfMemory ? DTP_ERR_NO_MEMORY : DTP_ERR_HIP,
            "workspace of %lld bytes: %s", (long long)need, hipGetErrorString(e));
  base = owned;
  return DTP_OK;
}

Workspace::~Workspace() {
  if (owned) (void)stream_free(owned, s);
}

size_t product_bytes(const Product& p) {
  if (p.N == 0 || p.K == 0) return 0;  // no tokens: nothing is launched
  return p.dtype == DTP_BF16 ? product_bytes_bf16(p) : product_bytes_f32(p);
}

dtp_status launch_product(const Product& p, char* workspace, hipStream_t s) {
  return p.dtype == DTP_BF16 ? launch_product_bf16(p, workspace, s) : launch_product_f32(p, workspace, s);
}

namespace {

// dz = scale act'(z) dy (linear), or dg = dh u act'(g) and du = dh act(g) (gated, `pre` [T][2][N]),
// rounded to the layer's type: dz [T][parts * ld], zeros from column N on.  One thread per 16 bytes
// of a part's row.  Bound by memory: 65,536 x 2 x 3,072 in bf16, 2.8 GB, in 517 us, 5.4 TB/s.
template <typename S, bool GATED>
__global__ void __launch_bounds__(256)
activation_grad_kernel(const S* __restrict__ dy, const float* __restrict__ pre, int act, float scale, int64_t T, int N,
                       int ld, S* __restrict__ dz) {
  constexpr int W = Elem<S>::kWide;
  const int pieces = ld / W;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < T * pieces; i += (int64_t)gridDim.x * 256) {
    const int64_t t = i / pieces;
    const int n = (int)(i - t * pieces) * W, count = N - n;
    float g[W] = {}, u[W] = {}, d[W] = {};
    if (count > 0) {
      load_row(dy + t * N + n, count, d);
      if (pre) load_row(pre + (GATED ? 2 : 1) * t * N + n, count, g);
      if (GATED) load_row(pre + (2 * t + 1) * N + n, count, u);
    }
#pragma unroll
    for (int e = 0; e < W; ++e) {
      float a, da;
      activate_grad<S>(act, g[e], a, da);
      if (e >= count) a = da = 0.0f;
      if (GATED) {
        g[e] = d[e] * u[e] * da;
        u[e] = d[e] * a;
      } else {
        g[e] = scale * d[e] * da;
      }
    }
    S* out = dz + t * (GATED ? 2 : 1) * ld + n;
    store_row(out, W, g);
    if (GATED) store_row(out + ld, W, u);
  }
}

constexpr int kSumCols = 256;

// partial[c][n] = sum over the rows of chunk c of scale act'(z) dy, unrounded.  A block: 256 columns
// in 32 groups of 8, times 8 rows at a time.
template <typename S>
__global__ void __launch_bounds__(256)
column_sums_kernel(const S* __restrict__ dy, const float* __restrict__ pre, int act, float scale, int64_t T, int N,
                   int64_t rows, float* __restrict__ partial) {
  __shared__ float sums[8][kSumCols];
  const int group = threadIdx.x % 32, lane = threadIdx.x / 32;
  const int n = blockIdx.x * kSumCols + 8 * group, count = N - n;
  const int64_t t0 = blockIdx.y * rows, t1 = t0 + rows < T ? t0 + rows : T;
  float acc[8] = {};
  if (count > 0)
    for (int64_t t = t0 + lane; t < t1; t += 8) {
      float d[8], z[8];
      load_row(dy + t * N + n, count, d);
      if (act != DTP_ACT_NONE) load_row(pre + t * N + n, count, z);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float a, da = 1.0f;
        if (act != DTP_ACT_NONE) activate_grad<S>(act, e < count ? z[e] : 0.0f, a, da);
        acc[e] += d[e] * da;
      }
    }
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[lane][8 * group + e] = scale * acc[e];
  __syncthreads();
  const int col = blockIdx.x * kSumCols + threadIdx.x;
  if (col >= N) return;
  float v = 0.0f;
#pragma unroll
  for (int l = 0; l < 8; ++l) v += sums[l][threadIdx.x];
  partial[(int64_t)blockIdx.y * N + col] = v;
}

// A block: 32 columns, their chunks dealt to eight threads each and summed in 64 bits.
template <typename S>
__global__ void __launch_bounds__(256)
join_sums_kernel(const float* __restrict__ partial, int chunks, int N, S* __restrict__ out) {
  __shared__ double sums[8][32];
  const int col = threadIdx.x % 32, lane = threadIdx.x / 32, n = blockIdx.x * 32 + col;
  double v = 0.0;
  if (n < N) {
#pragma unroll 8
    for (int c = lane; c < chunks; c += 8) v += (double)partial[(int64_t)c * N + n];
  }
  sums[lane][col] = v;
  __syncthreads();
  if (lane != 0 || n >= N) return;
#pragma unroll
  for (int l = 1; l < 8; ++l) v += sums[l][col];
  out[n] = Elem<S>::store((float)v);
}

template <typename S>
__global__ void __launch_bounds__(256) zeros_kernel(S* __restrict__ out, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) out[i] = S(0);
}

unsigned blocks_of(int64_t threads) { return (unsigned)std::min<int64_t>((threads + 255) / 256, 16384); }

dtp_status fill_zeros(void* p, int64_t n, int dtype, hipStream_t s) {
  if (dtype == DTP_BF16)
    zeros_kernel<<<blocks_of(n), 256, 0, s>>>((uint16_t*)p, n);
  else
    zeros_kernel<<<blocks_of(n), 256, 0, s>>>((float*)p, n);
  DTP_HIP(hipGetLastError());
  return DTP_OK;
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// Rows per chunk of a column sum, a multiple of the eight that a block takes at a time: 64, and fewer
// where that would be under a thousand blocks; at most 512 chunks.
int64_t sum_chunk_rows(int64_t T, int N) {
  const int64_t groups = (N + kSumCols - 1) / kSumCols;
  const int64_t rows = std::max<int64_t>(8, std::min<int64_t>(64, (T * groups / 1024 + 7) / 8 * 8));
  return std::max<int64_t>(rows, ((T + 511) / 512 + 7) / 8 * 8);
}
int64_t sum_chunks(int64_t T, int N) { return (T + sum_chunk_rows(T, N) - 1) / sum_chunk_rows(T, N); }

// dbias = sum over the tokens of scale act'(z) dy.
dtp_status launch_column_sums(const void* dy, const float* pre, int act, float scale, int64_t T, int N, int dtype,
                              void* out, float* partial, hipStream_t s) {
  const int chunks = (int)sum_chunks(T, N);
  const dim3 grid((N + kSumCols - 1) / kSumCols, chunks);
  if (dtype == DTP_BF16) {
    column_sums_kernel<<<grid, 256, 0, s>>>((const uint16_t*)dy, pre, act, scale, T, N, sum_chunk_rows(T, N),
                                            partial);
    join_sums_kernel<<<(N + 31) / 32, 256, 0, s>>>(partial, chunks, N, (uint16_t*)out);
  } else {
    column_sums_kernel<<<grid, 256, 0, s>>>((const float*)dy, pre, act, scale, T, N, sum_chunk_rows(T, N),
                                            partial);
    join_sums_kernel<<<(N + 31) / 32, 256, 0, s>>>(partial, chunks, N, (float*)out);
  }
  DTP_HIP(hipGetLastError());
  return DTP_OK;
}

template <bool GATED>
dtp_status launch_activation_grad(const void* dy, const float* pre, int act, float scale, int64_t T, int N, int ld,
                                  int dtype, void* dz, hipStream_t s) {
  if (dtype == DTP_BF16)
    activation_grad_kernel<uint16_t, GATED><<<blocks_of(T * (ld / 8)), 256, 0, s>>>(
        (const uint16_t*)dy, pre, act, scale, T, N, ld, (uint16_t*)dz);
  else
    activation_grad_kernel<float, GATED><<<blocks_of(T * (ld / 4)), 256, 0, s>>>(
        (const float*)dy, pre, act, scale, T, N, ld, (float*)dz);
  DTP_HIP(hipGetLastError());
  return DTP_OK;
}

// ---------------------------------------------------------------------------- plans
// A call's products and the offsets of its buffers in the workspace.  The pointers of `Product`s
// whose operand is a workspace buffer are set once the workspace is there.
struct Plan {
  size_t dz = 0, sums = 0, scratch = 0, bytes = 0;
  int ld = 0;  // of dz
};

size_t esize(int dtype) { return dtype == DTP_BF16 ? 2 : 4; }

Plan backward_plan(int64_t T, int K, int N, int parts, int dtype, bool pass, bool sums) {
  Plan w;
  w.ld = pass ? (int)pad32(N) : N;
  size_t at = 0;
  if (pass) at = up256(esize(dtype) * (size_t)T * parts * w.ld);
  w.sums = at;
  if (sums) at += up256(sizeof(float) * (size_t)sum_chunks(T, N) * N);
  w.scratch = at;
  w.bytes = at + std::max(product_bytes(dx_product(T, K, N, parts, w.ld, dtype)),
                          product_bytes(dw_product(T, K, N, parts, w.ld, dtype)));
  return w;
}

dtp_status check_sizes(int64_t T, int32_t K, int32_t N, int dtype) {
  DTP_CHECK(T >= 0, DTP_ERR_INVALID_ARG, "n_tokens=%lld is negative", (long long)T);
  DTP_CHECK(K > 0 && N > 0, DTP_ERR_INVALID_ARG, "every size must be positive (%d features in, %d out)", K, N);
  DTP_CHECK(T <= ((int64_t)1 << 30) && K <= (1 << 20) && N <= (1 << 20) && (int64_t)K * N <= ((int64_t)1 << 30),
            DTP_ERR_UNSUPPORTED, "shape too large (tokens <= 2^30, features <= 2^20, weights <= 2^30)");
  DTP_CHECK(dtype == DTP_BF16 || dtype == DTP_F32, DTP_ERR_UNSUPPORTED, "dtype %d", dtype);
  return DTP_OK;
}

int64_t workspace_bytes(ProductKind kind, int64_t T, int K, int N, int dtype, int act, bool backward) {
  const int parts = kind == kProductGated ? 2 : 1;
  size_t n = product_bytes(forward_product(kind, T, K, N, dtype));
  if (backward) n = std::max(n, backward_plan(T, K, N, parts, dtype, needs_pass(N, dtype, parts == 2, act != DTP_ACT_NONE),
                                       parts == 1).bytes);
  return (int64_t)n;
}

struct Weights {  // of a linear or a gated operator
  const void *w0, *w1;
};

dtp_status forward(ProductKind kind, int64_t T, int K, int N, int dtype, const void* x, Weights w, const void* bias,
                   const void* residual, int act, float alpha, void* y, float* pre, void* workspace,
                   int64_t given_bytes, hipStream_t s) {
  dtp_status st = check_sizes(T, K, N, dtype);
  if (st != DTP_OK || T == 0) return st;
  const bool gated = kind == kProductGated;
  DTP_CHECK(x && w.w0 && (w.w1 || !gated) && y, DTP_ERR_INVALID_ARG, "x, a weight or the output is NULL");
  const size_t es = esize(dtype), nx = es * T * K, nw = es * (size_t)N * K, ny = es * T * N;
  const Range in[] = {{x, nx, "x"}, {w.w0, nw, gated ? "w_gate" : "w"}, {w.w1, nw, "w_up"},
                      {bias, es * N, "bias"}, {residual, ny, "residual"}};
  const Range out[] = {{y, ny, gated ? "h" : "y", 16, 4}, {pre, sizeof(float) * T * N * (gated ? 2 : 1), "pre"},
                 {workspace, (size_t)std::max<int64_t>(given_bytes, 0), "workspace"}};
  if ((st = check_disjoint(out, 3, in, 5)) != DTP_OK || (st = check_ranges(in, 5)) != DTP_OK ||
      (st = check_ranges(out, 2)) != DTP_OK)
    return st;
  Product p = forward_product(kind, T, K, N, dtype);
  p.a0 = w.w0;
  p.a1 = w.w1;
  p.b = x;
  p.out.y = y;
  p.out.bias = bias;
  p.out.residual = residual;
  p.out.pre = pre;
  p.out.alpha = alpha;
  p.out.act = act;
  Workspace ws;
  if ((st = ws.open(workspace, given_bytes, (int64_t)product_bytes(p), s)) != DTP_OK) return st;
  return launch_product(p, ws.base, s);
}

// Both backward passes; w.w1 and dw1 are the up projection's.
dtp_status backward(ProductKind kind, int64_t T, int K, int N, int dtype, const void* x, Weights w, const void* dy,
                    int act, float alpha, const float* pre, void* dx, void* dw0, void* dw1, void* db, void* workspace,
                    int64_t given_bytes, hipStream_t s) {
  dtp_status st = check_sizes(T, K, N, dtype);
  if (st != DTP_OK) return st;
  const bool gated = kind == kProductGated, with_act = act != DTP_ACT_NONE;
  const int parts = gated ? 2 : 1;
  DTP_CHECK(!gated || (dw0 == nullptr) == (dw1 == nullptr), DTP_ERR_INVALID_ARG,
            "dw_gate and dw_up must be given together");
  if (!dx && !dw0 && !db) return DTP_OK;
  const size_t es = esize(dtype), nx = es * T * K, nw = es * (size_t)N * K, ny = es * T * N;
  if (T > 0) {
    DTP_CHECK(dy && (pre || !with_act), DTP_ERR_INVALID_ARG, "%s or pre is NULL", gated ? "dh" : "dy");
    DTP_CHECK(x || !dw0, DTP_ERR_INVALID_ARG, "x is NULL");
    DTP_CHECK((w.w0 && (w.w1 || !gated)) || !dx, DTP_ERR_INVALID_ARG, "a weight is NULL");
  }
  const Range in[] = {{T && dw0 ? x : nullptr, nx, "x"},
                      {T && dx ? w.w0 : nullptr, nw, gated ? "w_gate" : "w"},
                      {T && dx ? w.w1 : nullptr, nw, "w_up"},
                      {T ? dy : nullptr, ny, gated ? "dh" : "dy"},
                      {T && with_act ? pre : nullptr, sizeof(float) * T * N * parts, "pre"}};
  const Range out[] = {{T ? dx : nullptr, nx, "dx"}, {dw0, nw, gated ? "dw_gate" : "dw"}, {dw1, nw, "dw_up"},
                       {db, es * N, "dbias"}, {workspace, (size_t)std::max<int64_t>(given_bytes, 0), "workspace"}};
  if ((st = check_disjoint(out, 5, in, 5)) != DTP_OK || (st = check_ranges(in, 5)) != DTP_OK ||
      (st = check_ranges(out, 4)) != DTP_OK)
    return st;
  if (T == 0) {
    if (dw0 && (st = fill_zeros(dw0, (int64_t)N * K, dtype, s)) != DTP_OK) return st;
    if (dw1 && (st = fill_zeros(dw1, (int64_t)N * K, dtype, s)) != DTP_OK) return st;
    return db ? fill_zeros(db, N, dtype, s) : DTP_OK;
  }
  const bool pass = needs_pass(N, dtype, gated, with_act);
  const Plan plan = backward_plan(T, K, N, parts, dtype, pass, !gated);
  Workspace ws;
  if ((st = ws.open(workspace, given_bytes, (int64_t)plan.bytes, s)) != DTP_OK) return st;
  if (db &&
      (st = launch_column_sums(dy, pre, act, alpha, T, N, dtype, db, (float*)(ws.base + plan.sums), s)) != DTP_OK)
    return st;
  if (!dx && !dw0) return DTP_OK;
  const void* dz = dy;
  const float in_pass = with_act ? alpha : 1.0f;  // without an activation alpha is left to the products: dz is dy
  if (pass) {
    void* out_dz = ws.base + plan.dz;
    dz = out_dz;
    st = gated ? launch_activation_grad<true>(dy, pre, act, 1.0f, T, N, plan.ld, dtype, out_dz, s)
               : launch_activation_grad<false>(dy, with_act ? pre : nullptr, act, in_pass, T, N, plan.ld, dtype, out_dz, s);
    if (st != DTP_OK) return st;
  }
  char* scratch = ws.base + plan.scratch;
  if (dx) {
    Product p = dx_product(T, K, N, parts, plan.ld, dtype);
    p.a0 = w.w0;
    p.a1 = w.w1;
    p.b = dz;
    p.out.y = dx;
    p.out.alpha = with_act ? 1.0f : alpha;
    if ((st = launch_product(p, scratch, s)) != DTP_OK) return st;
  }
  if (dw0) {
    Product p = dw_product(T, K, N, parts, plan.ld, dtype);
    p.a0 = x;
    p.b = dz;
    p.out.y = dw0;
    p.out.y2 = dw1;
    p.out.alpha = with_act ? 1.0f : alpha;
    if ((st = launch_product(p, scratch, s)) != DTP_OK) return st;
  }
  return DTP_OK;
}

dtp_status check_act(int act, bool gated) {
  DTP_CHECK((act == DTP_ACT_NONE && !gated) || act == DTP_ACT_SILU || act == DTP_ACT_GELU, DTP_ERR_UNSUPPORTED,
            "activation %d", act);
  return DTP_OK;
}

}  // namespace
}  // namespace dtp

using namespace dtp;

extern "C" {

int64_t dtp_linear_workspace(int64_t n_tokens, int32_t n_in, int32_t n_out, dtp_dtype dtype, dtp_activation act,
                             int32_t backward) {
  int64_t n = -1;
  (void)guarded([&]() -> dtp_status {
    clear_error();
    dtp_status st;
    if ((st = check_act(act, false)) != DTP_OK || (st = check_sizes(n_tokens, n_in, n_out, dtype)) != DTP_OK) return st;
    n = workspace_bytes(kProductLinear, n_tokens, n_in, n_out, dtype, act, backward != 0);
    return DTP_OK;
  });
  return n;
}

int64_t dtp_gated_workspace(int64_t n_tokens, int32_t d_model, int32_t n_neurons, dtp_dtype dtype, int32_t backward) {
  int64_t n = -1;
  (void)guarded([&]() -> dtp_status {
    clear_error();
    const dtp_status st = check_sizes(n_tokens, d_model, n_neurons, dtype);
    if (st == DTP_OK) n = workspace_bytes(kProductGated, n_tokens, d_model, n_neurons, dtype, DTP_ACT_SILU, backward != 0);
    return st;
  });
  return n;
}

dtp_status dtp_linear_forward(int64_t n_tokens, int32_t n_in, int32_t n_out, dtp_dtype dtype, const void* x,
                              const void* w, const void* bias, const void* residual, dtp_activation act, float alpha,
                              void* y, float* pre, void* workspace, int64_t workspace_bytes, void* stream) {
  return guarded([&]() -> dtp_status {
    clear_error();
    const dtp_status st = check_act(act, false);
    if (st != DTP_OK) return st;
    DTP_CHECK(std::isfinite(alpha), DTP_ERR_INVALID_ARG, "alpha=%g must be finite", (double)alpha);
    return forward(kProductLinear, n_tokens, n_in, n_out, dtype, x, {w, nullptr}, bias, residual, act, alpha, y, pre,
                   workspace, workspace_bytes, (hipStream_t)stream);
  });
}

dtp_status dtp_linear_backward(int64_t n_tokens, int32_t n_in, int32_t n_out, dtp_dtype dtype, const void* x,
                               const void* w, const void* dy, dtp_activation act, float alpha, const float* pre,
                               void* dx, void* dw, void* dbias, void* workspace, int64_t workspace_bytes,
                               void* stream) {
  return guarded([&]() -> dtp_status {
    clear_error();
    const dtp_status st = check_act(act, false);
    if (st != DTP_OK) return st;
    DTP_CHECK(std::isfinite(alpha), DTP_ERR_INVALID_ARG, "alpha=%g must be finite", (double)alpha);
    return backward(kProductLinear, n_tokens, n_in, n_out, dtype, x, {w, nullptr}, dy, act, alpha, pre, dx, dw,
                    nullptr, dbias, workspace, workspace_bytes, (hipStream_t)stream);
  });
}

dtp_status dtp_gated_forward(int64_t n_tokens, int32_t d_model, int32_t n_neurons, dtp_dtype dtype, const void* x,
                             const void* w_gate, const void* w_up, dtp_activation act, void* h, float* pre,
                             void* workspace, int64_t workspace_bytes, void* stream) {
  return guarded([&]() -> dtp_status {
    clear_error();
    const dtp_status st = check_act(act, true);
    if (st != DTP_OK) return st;
    return forward(kProductGated, n_tokens, d_model, n_neurons, dtype, x, {w_gate, w_up}, nullptr, nullptr, act, 1.0f,
                   h, pre, workspace, workspace_bytes, (hipStream_t)stream);
  });
}

dtp_status dtp_gated_backward(int64_t n_tokens, int32_t d_model, int32_t n_neurons, dtp_dtype dtype, const void* x,
                              const void* w_gate, const void* w_up, dtp_activation act, const float* pre,
                              const void* dh, void* dx, void* dw_gate, void* dw_up, void* workspace,
                              int64_t workspace_bytes, void* stream) {
  return guarded([&]() -> dtp_status {
    clear_error();
    const dtp_status st = check_act(act, true);
    if (st != DTP_OK) return st;
    return backward(kProductGated, n_tokens, d_model, n_neurons, dtype, x, {w_gate, w_up}, dh, act, 1.0f, pre, dx,
                    dw_gate, dw_up, nullptr, workspace, workspace_bytes, (hipStream_t)stream);
  });
}

}  // extern "C"
