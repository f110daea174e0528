// Calls the entry points for prompts, shared prefixes and 4-bit weights with arguments that the host-side checks must reject (or accept as a no-op) before anything touches a GPU, in a build
// whose host code is compiled with -fsanitize=address,undefined. Needs no GPU. Prints "ok" and exits 0. Test infrastructure.
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/mlt.h"

#define CHECK(x) do { if (!(x)) { printf("failed: %s (line %d)\n", #x, __LINE__); return 1; } } while (0)

alignas(16) static uint16_t buf[64];        // stands in for device memory: never dereferenced
static void* const p = buf;
static void* const odd = reinterpret_cast<char*>(buf) + 2;
static const int32_t* const n = reinterpret_cast<const int32_t*>(buf);
static const uint8_t* const z = reinterpret_cast<const uint8_t*>(buf);
static const int64_t BIG = INT64_MAX / 2;

static int packed(int64_t T, int64_t B, int64_t Hq, int64_t H, int64_t D, int64_t ld, const void* q, float scale) {
  return mlt_mha_packed_fwd(T, T, B, Hq, H, D, q, ld, p, ld, p, ld, n, n, p, ld, scale, 1, MLT_BF16, nullptr);
}
static int prompt(int64_t T, int64_t B, int64_t Hq, int64_t H, int64_t D, int64_t block, int64_t max_blocks, int64_t ld, const void* q) {
  return mlt_paged_attn_prompt(T, B, Hq, H, D, block, max_blocks, 4, q, ld, p, p, n, n, n, p, ld, 1.f, MLT_FP16, nullptr);
}
static int prefix(int64_t B, int64_t Hq, int64_t H, int64_t D, int64_t block, int64_t max_blocks, int64_t len, const void* q, void* work, int64_t bytes) {
  return mlt_paged_attn_decode_prefix(B, Hq, H, D, block, max_blocks, 4, q, p, p, n, len, n, n, p, 1.f, work, bytes, MLT_BF16, nullptr);
}
static int gemm(int64_t M, int64_t N, int64_t K, int64_t lda, int64_t ldw, int64_t group, int64_t lds, const void* a, int dtype) {
  return mlt_gemm_w4(M, N, K, a, lda, p, ldw, group, p, lds, z, lds, p, N, dtype, nullptr);
}

int main() {
  CHECK(packed(-1, 1, 2, 1, 64, 128, p, 1.f) == MLT_ERR_INVALID_ARG);
  CHECK(packed(4, 1, 3, 2, 64, 192, p, 1.f) == MLT_ERR_INVALID_ARG);
  CHECK(packed(4, 1, 2, 1, 64, 120, p, 1.f) == MLT_ERR_INVALID_ARG);
  CHECK(packed(4, 1, 2, 1, 64, 128, odd, 1.f) == MLT_ERR_INVALID_ARG);
  CHECK(packed(4, 1, 2, 1, 64, 128, p, NAN) == MLT_ERR_INVALID_ARG);
  CHECK(packed(4, 1, 2, 1, 80, 160, p, 1.f) == MLT_ERR_UNSUPPORTED);
  CHECK(packed(BIG, 1, 2, 1, 64, 128, p, 1.f) == MLT_ERR_UNSUPPORTED);
  CHECK(packed(4, BIG, 2, 1, 64, 128, p, 1.f) == MLT_ERR_UNSUPPORTED);
  CHECK(packed(4, 1, BIG, BIG, 64, BIG, p, 1.f) == MLT_ERR_UNSUPPORTED);
  CHECK(packed(4, 1, 2, 1, 64, BIG - BIG % 8, p, 1.f) == MLT_ERR_UNSUPPORTED);
  CHECK(packed(0, 0, 0, 0, 64, 0, nullptr, 1.f) == MLT_OK);
  CHECK(prompt(4, 1, 2, 1, 128, 24, 4, 256, p) == MLT_ERR_UNSUPPORTED);
  CHECK(prompt(4, 1, 2, 1, 128, 16, BIG, 256, p) == MLT_ERR_UNSUPPORTED);
  CHECK(prompt(4, 1, 2, 1, 128, BIG - BIG % 16, 4, 256, p) == MLT_ERR_UNSUPPORTED);
  CHECK(prompt(4, BIG, 2, 1, 128, 16, 4, 256, p) == MLT_ERR_UNSUPPORTED);
  CHECK(prompt(4, 1, 2, 1, 128, 16, 4, 248, p) == MLT_ERR_INVALID_ARG);
  CHECK(prompt(4, 1, 2, 1, 128, 16, 4, 256, nullptr) == MLT_ERR_INVALID_ARG);
  CHECK(prefix(1, 2, 1, 64, 16, 4, 65, p, p, 0) == MLT_ERR_INVALID_ARG);
  CHECK(prefix(1, 2, 1, 64, 16, 4, BIG, p, p, 0) == MLT_ERR_INVALID_ARG);
  CHECK(prefix(1, 2, 1, 64, 16, 4, 30, p, odd, 64) == MLT_ERR_INVALID_ARG);
  CHECK(prefix(1, 2, 1, 64, 16, 4, 30, p, p, -1) == MLT_ERR_INVALID_ARG);
  CHECK(prefix(BIG, 2, 1, 64, 16, 4, 30, p, p, 0) == MLT_ERR_UNSUPPORTED);
  CHECK(prefix(4, BIG, BIG, 64, 16, 4, 30, p, p, 0) == MLT_ERR_UNSUPPORTED);
  CHECK(prefix(0, 2, 1, 64, 16, 4, 30, nullptr, nullptr, 0) == MLT_OK);
  CHECK(mlt_paged_attn_decode_prefix_work(BIG, 2, 1, 64, 16, 4, 30) == MLT_ERR_UNSUPPORTED);
  CHECK(mlt_paged_attn_decode_prefix_work(1, 2, 1, 64, 16, BIG, 30) < 0);
  CHECK(gemm(4, 4, 64, 64, 32, 128, 4, p, 7) == MLT_ERR_INVALID_ARG);
  CHECK(gemm(4, 4, 64, 64, 32, 100, 4, p, MLT_BF16) == MLT_ERR_UNSUPPORTED);
  CHECK(gemm(4, 4, 64, 56, 32, 128, 4, p, MLT_BF16) == MLT_ERR_INVALID_ARG);
  CHECK(gemm(4, 4, 64, 64, 32, 128, 3, p, MLT_BF16) == MLT_ERR_INVALID_ARG);
  CHECK(gemm(4, 4, 64, 64, 32, 128, 4, odd, MLT_BF16) == MLT_ERR_INVALID_ARG);
  CHECK(gemm(4, 4, 48, 64, 32, 32, 4, p, MLT_BF16) == MLT_ERR_UNSUPPORTED);
  CHECK(gemm(4, 4, 64, 1 << 23, 32, 128, 4, p, MLT_BF16) == MLT_ERR_UNSUPPORTED);
  CHECK(gemm(4, 4, 64, 64, 1 << 24, 128, 4, p, MLT_BF16) == MLT_ERR_UNSUPPORTED);
  CHECK(gemm(4, 4, 64, 64, 32, 128, 1 << 26, p, MLT_BF16) == MLT_ERR_UNSUPPORTED);
  CHECK(gemm(BIG, 4, 64, 64, 32, 128, 4, p, MLT_FP16) == MLT_ERR_UNSUPPORTED);
  CHECK(gemm(4, BIG, 64, 64, 32, 128, BIG, p, MLT_FP16) == MLT_ERR_UNSUPPORTED);
  CHECK(gemm(4, 4, BIG - BIG % 64, BIG - BIG % 64, BIG / 2 + 1, 128, 4, p, MLT_FP16) == MLT_ERR_UNSUPPORTED);
  CHECK(gemm(0, 4, 64, 0, 0, 128, 0, nullptr, MLT_FP16) == MLT_OK);
  printf("ok\n");
  return 0;
}
