// The launches that dense_plan.h chooses, from the header that the library's own calls use.  One
// line in, "linear|gated tokens in out bf16|f32 act", gives one line per product out:
//   forward|dx|dw  tile rows x columns (0 x 0: streamed)  splits  stages  stages per split  tiles
//   threads of the largest launch, along its longest axis
// The argument: compute units of the GPU, 256 without it.
#include <cstdio>
#include <cstring>

#include "dense_plan.h"

using namespace dtp;

static int cus = 256;

static void print(const char* name, const Product& p, bool first) {
  long long m, n, splits, stages, per, tiles, threads;
  const long long planes = p.kind == kProductGated ? 2 : 1;
  bool stream;
  if (p.dtype == DTP_BF16) {
    const ShapeBf16 s = choose_bf16(p, cus);
    const Tile& t = kTilesBf16[s.tile];
    stream = s.stream, splits = s.splits, stages = s.nq, per = s.per, m = t.m, n = t.n;
    tiles = (planes * p.M + m - 1) / m * ((p.N + n - 1) / n);
    threads = (tiles * splits < t.per_cu * cus ? tiles * splits : t.per_cu * cus) * 512;
  } else {
    const ShapeF32 s = choose_f32(p, cus);
    stream = s.stream, splits = s.splits, stages = (long long)s.stages * p.segments, per = s.per;
    m = n = 64 * s.f;
    tiles = (long long)s.m_tiles * s.n_tiles;
    threads = stream ? 0 : (long long)s.launch_tiles(0) * s.threads();
  }
  if (stream) m = n = tiles = 0, threads = (p.M + 15) / 16 * 512;
  std::printf("%s%s %lld %lld %lld %lld %lld %lld %lld", first ? "" : " ", name, m, n, splits, stages, per, tiles, threads);
}

int main(int argc, char** argv) {
  if (argc > 1) std::sscanf(argv[1], "%d", &cus);
  char kind[16], type[16];
  long long T;
  int K, N, act;
  while (std::scanf("%15s %lld %d %d %15s %d", kind, &T, &K, &N, type, &act) == 6) {
    const bool gated = !std::strcmp(kind, "gated");
    const int dtype = !std::strcmp(type, "bf16") ? DTP_BF16 : DTP_F32, parts = gated ? 2 : 1;
    const int ld = needs_pass(N, dtype, gated, act != DTP_ACT_NONE) ? (int)pad32(N) : N;
    print("forward", forward_product(gated ? kProductGated : kProductLinear, T, K, N, dtype), true);
    print("dx", dx_product(T, K, N, parts, ld, dtype), false);
    print("dw", dw_product(T, K, N, parts, ld, dtype), false);
    std::printf("\n");
  }
  return 0;
}
