// The products of the dense operators, of any type, layout and size: tiles of 64 x 64 through
// LDS, fp32 multiply-adds.
#include "dense.h"

namespace dtp {
namespace {

constexpr int kST = 64, kSK = 16;

template <typename S, ProductKind KIND>
__global__ void __launch_bounds__(256) simple_product_kernel(Product p) {
  __shared__ float a_tile[2][kSK][kST + 1], b_tile[kSK][kST + 1];
  const int m0 = blockIdx.x * kST, tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  const int64_t n0 = (int64_t)blockIdx.y * kST;
  float acc[2][4][4] = {};
  for (int seg = 0; seg < p.segments; ++seg)
    for (int64_t k0 = 0; k0 < p.K; k0 += kSK) {
      __syncthreads();
      for (int i = threadIdx.x; i < kST * kSK; i += 256) {
        const int ar = p.at ? i % kST : i / kSK, ak = p.at ? i / kST : i % kSK;
        const int br = p.bt ? i % kST : i / kSK, bk = p.bt ? i / kST : i % kSK;
        const int64_t m = m0 + ar, ka = k0 + ak, n = n0 + br, kb = k0 + bk;
        const bool in_a = m < p.M && ka < p.K, in_b = n < p.N && kb < p.K;
        const int64_t ao = p.at ? ka * p.lda + m : m * p.lda + ka;
        const int64_t bo = (p.bt ? kb * p.ldb + n : n * p.ldb + kb) + seg * p.b_seg;
        a_tile[0][ak][ar] = in_a ? Elem<S>::load(((const S*)(seg ? p.a1 : p.a0))[ao]) : 0.0f;
        if constexpr (KIND == kProductGated) a_tile[1][ak][ar] = in_a ? Elem<S>::load(((const S*)p.a1)[ao]) : 0.0f;
        b_tile[bk][br] = in_b ? Elem<S>::load(((const S*)p.b)[bo]) : 0.0f;
      }
      __syncthreads();
      for (int k = 0; k < kSK; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            acc[0][j][i] = fmaf(a_tile[0][k][4 * tx + i], b_tile[k][4 * ty + j], acc[0][j][i]);
            if constexpr (KIND == kProductGated)
              acc[1][j][i] = fmaf(a_tile[1][k][4 * tx + i], b_tile[k][4 * ty + j], acc[1][j][i]);
          }
    }
  ProductOut o = p.out;
  o.vec = false;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (n0 + 4 * ty + j < p.N) write_product<S, KIND, 4>(o, n0 + 4 * ty + j, m0 + 4 * tx, p.M, acc[0][j], acc[1][j]);
}

template <typename S>
void launch(const Product& p, hipStream_t s) {
  const dim3 grid((p.M + kST - 1) / kST, (unsigned)((p.N + kST - 1) / kST));
  switch (p.kind) {
    case kProductLinear: simple_product_kernel<S, kProductLinear><<<grid, 256, 0, s>>>(p); break;
    case kProductGated: simple_product_kernel<S, kProductGated><<<grid, 256, 0, s>>>(p); break;
    case kProductGrad: simple_product_kernel<S, kProductGrad><<<grid, 256, 0, s>>>(p); break;
  }
}

}  // namespace

size_t product_bytes(const Product& p) { return p.dtype == DTP_BF16 ? product_bytes_bf16(p) : 0; }

dtp_status launch_product(const Product& p, char* workspace, hipStream_t s) {
  if (p.N == 0) return DTP_OK;
  if (p.dtype == DTP_BF16) return launch_product_bf16(p, workspace, s);
  launch<float>(p, s);
  DTP_HIP(hipGetLastError());
  return DTP_OK;
}

}  // namespace dtp
