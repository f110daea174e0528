// Asks the 8-bit operators for launches of more than 2^32 work-items. All of them have to be refused before anything touches a device (the pointers lead nowhere).
// Prints one status a line. Test infrastructure.
#include <stdio.h>

#include "../../include/mlt.h"
#include "../../paper_2503_14985_amd/csrc/mlt_internal.h"

using namespace mlt;

static uint16_t* const P = reinterpret_cast<uint16_t*>(0x100000);
static uint8_t* const P8 = reinterpret_cast<uint8_t*>(P);
static float* const F = reinterpret_cast<float*>(P);
static const int32_t* const I = reinterpret_cast<const int32_t*>(P);

static int quant(int64_t M, int64_t K, int64_t rows) { return run_quant(QuantArgs{M, K, P, K, rows, P8, K, F, M, MLT_BF16}, nullptr); }
static int gemm(int64_t M, int64_t N, int forced, int parts) {
  char name[128];
  return run_gemm_fp8(GemmFp8Args{M, N, 2048, P8, 2048, F, M, P8, 2048, F, N, P, N, MLT_FP16, forced, parts}, nullptr, name, sizeof name);
}
static int append(int64_t T, int64_t Hq, int64_t H, int64_t block, bool fp8) {
  AppendArgs a{T, 1, Hq, H, 64, block, 1 << 20, 1 << 20, P, 64 * Hq, P, 64 * H, P, 64 * H, I, I, I, nullptr, nullptr, 0, 0, 0, P, P, P, F, F, MLT_BF16};
  return run_append(a, fp8, nullptr);
}
static int attention(int64_t B, int64_t Hq, int64_t H, int split) {
  int n, w;
  return run_paged_fp8(PagedFp8Args{B, Hq, H, 64, 16, 4096, 4096, P, P8, P8, F, F, I, I, P, 1.f, MLT_FP16, split}, nullptr, &n, &w);
}

int main() {
  const int64_t most = ((int64_t)1 << 24) - 1;            // workgroups of 256
  printf("%d\n", quant(most * 16 + 1, 512, 1));
  printf("%d\n", quant(16, most * 512 + 8, 1));
  printf("%d\n", quant(most / 2 * 128 + 1, 384, 128));
  printf("%d\n", gemm((int64_t)1 << 30, 384, GEMM_AUTO, 0));
  printf("%d\n", gemm((int64_t)1 << 30, 384, GEMM_128_KP, 8));
  printf("%d\n", gemm(8192, (int64_t)1 << 30, GEMM_SKINNY, 2));
  printf("%d\n", append(most * 4 + 1, 1, 0, 16, false));
  printf("%d\n", append(most * 4 + 1, 1, 1, 16, true));
  printf("%d\n", append((int64_t)1 << 30, 0, 64, 1024, true));
  printf("%d\n", attention(most + 1, 1, 1, 0));
  printf("%d\n", attention(1 << 20, 32, 16, 9));
  printf("%d\n", attention(1 << 20, 17 * 8, 8, 1));
  return 0;
}
