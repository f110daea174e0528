// Asks the operators for prompts, shared prefixes and 4-bit weights for launches of more than 2^32 work-items. All of them have to be refused before anything touches a device (the pointers
// lead nowhere). Prints one status a line. Test infrastructure.
#include <stdio.h>

#include "../../include/mlt.h"
#include "../../paper_2503_14985_amd/csrc/mlt_internal.h"

using namespace mlt;

static uint16_t* const P = reinterpret_cast<uint16_t*>(0x100000);
static uint8_t* const P8 = reinterpret_cast<uint8_t*>(P);
static const int32_t* const I = reinterpret_cast<const int32_t*>(P);
static char name[128];

static int prompt(int64_t T, int64_t B, int64_t Hq, int64_t H, int64_t D, bool paged, int causal) {
  PromptArgs a{T, T, B, Hq, H, D, P, Hq * D, P, H * D, P, H * D, I, I, paged ? 16 : 0, paged ? 4 : 0, paged ? 64 : 0, paged ? I : nullptr, paged ? I : nullptr, P, Hq * D, 1.f, causal, MLT_BF16};
  return run_prompt(a, nullptr, name, sizeof name);
}
static int prefix(int64_t B, int64_t Hq, int64_t H, int64_t D, int64_t len) {
  PrefixArgs a{B, Hq, H, D, 16, 4, 64, P, P, P, I, len, I, I, P, 1.f, nullptr, 0, MLT_FP16};
  return run_paged_prefix(a, nullptr, name, sizeof name);
}
static int gemm(int64_t M, int64_t N, int64_t K, bool zeros) {
  Gemm4bitArgs a{M, N, K, P, K, P8, K / 2, 128, P, N, zeros ? P8 : nullptr, N, P, N, MLT_BF16};
  return run_gemm_4bit(a, nullptr, name, sizeof name);
}

int main() {
  printf("%d\n", prompt(1 << 30, 4, 4, 1, 64, false, 1));
  printf("%d\n", prompt(1 << 30, 4, 8, 8, 128, false, 0));
  printf("%d\n", prompt(1 << 20, 1 << 23, 4, 4, 128, true, 1));
  printf("%d\n", prefix(1 << 24, 16, 16, 64, 0));
  printf("%d\n", prefix(1 << 24, 16, 16, 128, 30));
  printf("%d\n", prefix(1 << 22, 64, 64, 128, 64));
  printf("%d\n", gemm(1 << 23, 1 << 20, 256, false));
  printf("%d\n", gemm(1 << 20, 1 << 20, 4096, true));
  return 0;
}
