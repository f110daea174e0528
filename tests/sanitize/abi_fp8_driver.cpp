// Calls the 8-bit entry points of the C ABI with arguments that the host-side checks must reject (or accept as a no-op) before anything touches a GPU, in a build
// whose host code is compiled with -fsanitize=address,undefined. Needs no GPU. Prints "ok" and exits 0. Test infrastructure.
#include <limits.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/mlt.h"
#include "../../include/mlt_diag.h"

#define CHECK(x) do { if (!(x)) { printf("failed: %s (line %d)\n", #x, __LINE__); return 1; } } while (0)

alignas(16) static uint16_t buf[64];        // stands in for device memory: never dereferenced
static void* const p = buf;
static void* const odd = reinterpret_cast<char*>(buf) + 2;
static float* const f = reinterpret_cast<float*>(buf);
static const int32_t* const n = reinterpret_cast<const int32_t*>(buf);
static const int64_t BIG = INT64_MAX / 2;

static int append(int64_t T, int64_t B, int64_t Hq, int64_t H, int64_t D, int64_t block, int64_t ld, int64_t rot, const void* q, const int32_t* offsets, bool fp8, float* ks) {
  if (fp8)
    return mlt_paged_append_fp8(T, B, Hq, H, D, block, 4, 4, q, ld, p, ld, p, ld, offsets, n, n, f, f, rot, 16, 0, p, p, p, ks, f, MLT_BF16, nullptr);
  return mlt_paged_append(T, B, Hq, H, D, block, 4, 4, q, ld, p, ld, p, ld, offsets, n, n, f, f, rot, 16, 1, p, p, p, MLT_FP16, nullptr);
}
static int attn(int64_t B, int64_t Hq, int64_t H, int64_t D, int64_t block, int64_t max_blocks, int64_t num_blocks, const void* q, float scale, int dtype) {
  return mlt_paged_attn_decode_fp8(B, Hq, H, D, block, max_blocks, num_blocks, q, p, p, f, f, n, n, p, scale, dtype, nullptr);
}

int main() {
  // quantisation: types, sizes, blocks, leading dimensions, alignment, no-ops
  CHECK(mlt_quant_fp8(4, 128, p, 128, 1, p, 128, f, 4, 9, nullptr) == MLT_ERR_INVALID_ARG);
  CHECK(mlt_quant_fp8(-1, 128, p, 128, 1, p, 128, f, 4, MLT_BF16, nullptr) == MLT_ERR_INVALID_ARG);
  CHECK(mlt_quant_fp8(4, 128, p, 128, 0, p, 128, f, 4, MLT_BF16, nullptr) == MLT_ERR_INVALID_ARG);
  CHECK(mlt_quant_fp8(4, 128, p, 128, 64, p, 128, f, 4, MLT_BF16, nullptr) == MLT_ERR_UNSUPPORTED);
  CHECK(mlt_quant_fp8(4, 128, nullptr, 128, 1, p, 128, f, 4, MLT_BF16, nullptr) == MLT_ERR_INVALID_ARG);
  CHECK(mlt_quant_fp8(4, 128, p, 120, 1, p, 128, f, 4, MLT_BF16, nullptr) == MLT_ERR_INVALID_ARG);
  CHECK(mlt_quant_fp8(4, 128, p, 128, 1, p, 128, f, 3, MLT_BF16, nullptr) == MLT_ERR_INVALID_ARG);
  CHECK(mlt_quant_fp8(4, 128, odd, 128, 1, p, 128, f, 4, MLT_BF16, nullptr) == MLT_ERR_INVALID_ARG);
  CHECK(mlt_quant_fp8(4, 132, p, 136, 1, p, 144, f, 4, MLT_BF16, nullptr) == MLT_ERR_UNSUPPORTED);
  CHECK(mlt_quant_fp8(4, 128, p, 132, 1, p, 128, f, 4, MLT_BF16, nullptr) == MLT_ERR_UNSUPPORTED);
  CHECK(mlt_quant_fp8(BIG, 128, p, 128, 1, p, 128, f, BIG, MLT_BF16, nullptr) == MLT_ERR_UNSUPPORTED);
  CHECK(mlt_quant_fp8(4, BIG, p, BIG, 128, p, BIG, f, 4, MLT_FP16, nullptr) == MLT_ERR_UNSUPPORTED);
  CHECK(mlt_quant_fp8(0, 128, nullptr, 0, 1, nullptr, 0, nullptr, 0, MLT_BF16, nullptr) == MLT_OK);
  CHECK(mlt_quant_fp8(4, 0, nullptr, 0, 128, nullptr, 0, nullptr, 0, MLT_FP16, nullptr) == MLT_OK);
  // product
  CHECK(mlt_gemm_fp8(4, 4, 128, p, 128, f, 4, p, 128, f, 1, p, 4, 3, nullptr) == MLT_ERR_INVALID_ARG);
  CHECK(mlt_gemm_fp8(4, -4, 128, p, 128, f, 4, p, 128, f, 1, p, 4, MLT_BF16, nullptr) == MLT_ERR_INVALID_ARG);
  CHECK(mlt_gemm_fp8(4, 4, 128, p, 128, nullptr, 4, p, 128, f, 1, p, 4, MLT_BF16, nullptr) == MLT_ERR_INVALID_ARG);
  CHECK(mlt_gemm_fp8(4, 4, 128, p, 128, f, 3, p, 128, f, 1, p, 4, MLT_BF16, nullptr) == MLT_ERR_INVALID_ARG);
  CHECK(mlt_gemm_fp8(4, 129, 128, p, 128, f, 4, p, 128, f, 1, p, 129, MLT_BF16, nullptr) == MLT_ERR_INVALID_ARG);
  CHECK(mlt_gemm_fp8(4, 4, 128, p, 128, f, 4, p, 128, f, 1, p, 3, MLT_BF16, nullptr) == MLT_ERR_INVALID_ARG);
  CHECK(mlt_gemm_fp8(4, 4, 128, odd, 128, f, 4, p, 128, f, 1, p, 4, MLT_BF16, nullptr) == MLT_ERR_INVALID_ARG);
  CHECK(mlt_gemm_fp8(4, 4, 120, p, 128, f, 4, p, 128, f, 1, p, 4, MLT_BF16, nullptr) == MLT_ERR_UNSUPPORTED);
  CHECK(mlt_gemm_fp8(4, 4, 128, p, 136, f, 4, p, 128, f, 1, p, 4, MLT_BF16, nullptr) == MLT_ERR_UNSUPPORTED);
  CHECK(mlt_gemm_fp8(4, 4, 128, p, (int64_t)1 << 24, f, 4, p, 128, f, 1, p, 4, MLT_BF16, nullptr) == MLT_ERR_UNSUPPORTED);
  CHECK(mlt_gemm_fp8(BIG, 4, 128, p, 128, f, BIG, p, 128, f, 1, p, 4, MLT_BF16, nullptr) == MLT_ERR_UNSUPPORTED);
  CHECK(mlt_gemm_fp8(0, 4, 128, nullptr, 0, nullptr, 0, nullptr, 0, nullptr, 0, nullptr, 0, MLT_BF16, nullptr) == MLT_OK);
  // append: both forms
  for (int fp8 = 0; fp8 < 2; ++fp8) {
    CHECK(append(-1, 1, 1, 1, 64, 16, 64, 0, p, n, fp8, f) == MLT_ERR_INVALID_ARG);
    CHECK(append(1, 1, 1, 1, 96, 16, 96, 0, p, n, fp8, f) == MLT_ERR_UNSUPPORTED);
    CHECK(append(1, 1, 1, 1, 64, 24, 64, 0, p, n, fp8, f) == MLT_ERR_UNSUPPORTED);
    CHECK(append(1, 1, 1, 1, 64, 16, 64, 24, p, n, fp8, f) == MLT_ERR_UNSUPPORTED);
    CHECK(append(1, 1, 1, 1, 64, 16, 64, 128, p, n, fp8, f) == MLT_ERR_INVALID_ARG);
    CHECK(append(1, 1, 1, 1, 64, 16, 64, 64, nullptr, n, fp8, f) == MLT_ERR_INVALID_ARG);
    CHECK(append(1, 1, 1, 1, 64, 16, 64, 64, odd, n, fp8, f) == MLT_ERR_INVALID_ARG);
    CHECK(append(1, 1, 2, 1, 64, 16, 64, 64, p, n, fp8, f) == MLT_ERR_INVALID_ARG);
    CHECK(append(1, 1, 1, 1, 64, 16, 68, 64, p, n, fp8, f) == MLT_ERR_UNSUPPORTED);
    CHECK(append(1, 1, 1, 1, 64, 16, 64, 64, p, nullptr, fp8, f) == MLT_ERR_INVALID_ARG);
    CHECK(append(BIG, 1, 1, 1, 64, 16, 64, 64, p, n, fp8, f) == MLT_ERR_UNSUPPORTED);
    CHECK(append(1, 1, BIG, 1, 64, 16, BIG, 64, p, n, fp8, f) == MLT_ERR_UNSUPPORTED);
    CHECK(append(0, 1, 1, 1, 64, 16, 64, 64, nullptr, nullptr, fp8, nullptr) == MLT_OK);
  }
  CHECK(append(1, 1, 1, 1, 64, 16, 64, 64, p, n, true, nullptr) == MLT_ERR_INVALID_ARG);
  // attention
  CHECK(attn(1, 1, 1, 96, 16, 1, 1, p, 1.f, MLT_BF16) == MLT_ERR_UNSUPPORTED);
  CHECK(attn(1, 1, 1, 64, 24, 1, 1, p, 1.f, MLT_BF16) == MLT_ERR_UNSUPPORTED);
  CHECK(attn(1, 1, 1, 64, 2048, 1, 1, p, 1.f, MLT_BF16) == MLT_ERR_UNSUPPORTED);
  CHECK(attn(1, 3, 2, 64, 16, 1, 1, p, 1.f, MLT_BF16) == MLT_ERR_INVALID_ARG);
  CHECK(attn(1, 1, 0, 64, 16, 1, 1, p, 1.f, MLT_BF16) == MLT_ERR_INVALID_ARG);
  CHECK(attn(1, 1, 1, 64, 16, 0, 1, p, 1.f, MLT_BF16) == MLT_ERR_INVALID_ARG);
  CHECK(attn(1, 1, 1, 64, 16, 1, 1, nullptr, 1.f, MLT_BF16) == MLT_ERR_INVALID_ARG);
  CHECK(attn(1, 1, 1, 64, 16, 1, 1, odd, 1.f, MLT_BF16) == MLT_ERR_INVALID_ARG);
  CHECK(attn(1, 1, 1, 64, 16, 1, 1, p, 1.f / 0.f, MLT_BF16) == MLT_ERR_INVALID_ARG);
  CHECK(attn(1, 1, 1, 64, 16, 1, 1, p, 1.f, 4) == MLT_ERR_INVALID_ARG);
  CHECK(attn(1, 1, 1, 64, 16, INT_MAX / 16, 1, p, 1.f, MLT_BF16) == MLT_ERR_UNSUPPORTED);
  CHECK(attn(1, 8, 8, 64, 1024, 1, INT_MAX / 256, p, 1.f, MLT_BF16) == MLT_ERR_UNSUPPORTED);
  CHECK(attn((int64_t)1 << 30, 8, 8, 64, 16, 1, 1, p, 1.f, MLT_BF16) == MLT_ERR_UNSUPPORTED);
  CHECK(attn(0, 8, 8, 64, 16, 1, 1, nullptr, 1.f, MLT_BF16) == MLT_OK);
  printf("ok\n");
  return 0;
}
