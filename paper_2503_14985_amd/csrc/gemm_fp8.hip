// C = A * B^T on e4m3 operands with a scale for each block of 128 of K (mlt_gemm_fp8):
//   C[m][n] = sum over blocks kb of Sa[kb][m] * Sb[kb][n / 128] * sum over k in kb of A[m][k] * B[n][k]
// One MFMA (16x16x128) multiplies a block's 128 k of a 16 x 16 tile; its fp32 result, started from zero, goes into the fp32
// accumulator with the product of the two scales.
#include "fp8.h"
#include "mlt_internal.h"

namespace mlt {

namespace {

// The plain form: fragments straight from memory, a wavefront 16 rows x 64 columns, a workgroup 64 x 64.
template <typename Tag>
__global__ __launch_bounds__(256) void gemm_fp8_direct_kernel(int M, int N, int K, const uint8_t* __restrict__ A, int64_t lda, const float* __restrict__ Sa, int64_t ldsa,
                                                              const uint8_t* __restrict__ B, int64_t ldb, const float* __restrict__ Sb, int64_t ldsb,
                                                              uint16_t* __restrict__ C, int64_t ldc) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4;
  const int m0 = (int)blockIdx.y * 64 + wave * 16, n0 = (int)blockIdx.x * 64;
  if (m0 >= M) return;
  const u32x4 zero4 = {0u, 0u, 0u, 0u};
  const int m = m0 + r16 < M ? m0 + r16 : M - 1;
  const uint8_t* ap = A + (int64_t)m * lda;
  f32x4 acc[4] = {};
  for (int kb = 0; kb * F8_KB < K; ++kb) {
    const int k = kb * F8_KB + 32 * g;
    auto piece = [&](const uint8_t* row, int at) { return at < K ? *reinterpret_cast<const u32x4_mem*>(row + at) : zero4; };
    const u32x4 a0 = piece(ap, k), a1 = piece(ap, k + 16);
    const float sa = Sa[(int64_t)kb * ldsa + m];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + 16 * j + r16 < N ? n0 + 16 * j + r16 : N - 1;
      const uint8_t* bp = B + (int64_t)n * ldb;
      const f32x4 part = mfma16_e4m3(piece(bp, k), piece(bp, k + 16), a0, a1, f32x4{0.f, 0.f, 0.f, 0.f});
      const float s = sa * Sb[(int64_t)kb * ldsb + n0 / F8_KB];
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[j][r] += part[r] * s;
    }
  }
  if (m0 + r16 >= M) return;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int n = n0 + 16 * j + 4 * g + r;
      if (n < N) C[(int64_t)m * ldc + n] = Elem<Tag>::from_f32(acc[j][r]);
    }
}

}  // namespace

int run_gemm_fp8(const GemmFp8Args& a, hipStream_t s, const char** name) {
  *name = "gemm_fp8_64x64_direct";
  auto kern = a.dtype == MLT_BF16 ? gemm_fp8_direct_kernel<bf16_tag> : gemm_fp8_direct_kernel<f16_tag>;
  hipLaunchKernelGGL(kern, dim3((unsigned)((a.N + 63) / 64), (unsigned)((a.M + 63) / 64)), dim3(256), 0, s, (int)a.M, (int)a.N, (int)a.K, a.A, a.lda, a.Sa, a.ldsa,
                     a.B, a.ldb, a.Sb, a.ldsb, a.C, a.ldc);
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

}  // namespace mlt
