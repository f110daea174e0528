// Asks the 16-bit operators for launches of more than 2^32 work-items. All of them have to be refused before anything touches a device (the pointers lead nowhere).
// Prints one status a line. Test infrastructure.
#include <stdio.h>

#include "../../include/mlt.h"
#include "../../paper_2503_14985_amd/csrc/mlt_internal.h"

using namespace mlt;

static uint16_t* const P = reinterpret_cast<uint16_t*>(0x100000);
static const int32_t* const I = reinterpret_cast<const int32_t*>(P);

static int gemm(int64_t M, int64_t N, int64_t K, int transB, int forced, int odd) {
  GemmArgs g{};
  g.M = M; g.N = N; g.K = K;
  g.A = P + odd; g.lda = K;
  g.B = P; g.ldb = transB ? K : N; g.transB = transB;
  g.C = P; g.ldc = N;
  g.forced = forced;
  GemmPlan p = plan_gemm(g);
  return run_gemm(g, p, nullptr);
}
static int mha(int64_t B, int64_t H, int64_t Sq, int64_t Sk, int64_t D, int causal, int forced) {
  MhaArgs a{B, H, Sq, Sk, D, P, P, P, P, 1.f, causal, MLT_BF16};
  a.forced = forced;
  MhaPlan p = plan_mha(a);
  return run_mha(a, p, nullptr);
}
static int paged(int64_t B, int64_t H, int64_t D) {
  PagedArgs a{};
  a.B = B; a.H = H; a.D = D; a.block_size = 16; a.max_blocks = 1; a.num_blocks = 16;
  a.Q = a.Kc = a.Vc = P; a.O = P; a.block_table = a.seq_lens = I;
  int n;
  return run_paged_decode(a, nullptr, &n);
}

int main() {
  const int64_t big = (int64_t)1 << 30;
  const int variants[] = {GEMM_AUTO, GEMM_256_PP16, GEMM_128_PP16, GEMM_256X128_KP, GEMM_128_KP, GEMM_256_W8, GEMM_128_W8, GEMM_64X128_W8, GEMM_64_W4, GEMM_128_K2, GEMM_64_K4};
  for (int v : variants) {
    printf("%d\n", gemm(big, 600, 64, 1, v, 0));
    printf("%d\n", gemm(big + 7, 601, 65, 0, v, 1));
  }
  printf("%d\n", gemm(big, 1100, 64, 1, GEMM_256_W4, 0));
  printf("%d\n", gemm(8, 2 * big - 64, 3, 0, GEMM_GENERAL, 1));
  const int kinds[] = {MHA_AUTO, MHA_PP32, MHA_PP16, MHA_K2, MHA_K4};
  for (int v : kinds) {
    printf("%d\n", mha(1 << 20, 16, 1, 1, 64, 0, v));
    printf("%d\n", mha(1 << 20, 8, 300, 300, 128, 1, v));
  }
  printf("%d\n", paged(1 << 20, 16, 64));
  printf("%d\n", paged(1 << 24, 1, 128));
  return 0;
}
