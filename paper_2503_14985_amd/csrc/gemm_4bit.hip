// Few rows times 4-bit weights with a scale for every group (mlt_gemm_w4): first form. A wavefront owns one element of C: a lane takes 8 weights at a
// time, the lanes' sums meet at the end.
#include <stdio.h>

#include "attn_rows.h"
#include "mlt_internal.h"

namespace mlt {

namespace {

template <typename Tag>
__global__ __launch_bounds__(256) void gemm_4bit_kernel(Gemm4bitArgs a) {
  const int64_t e = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
  if (e >= a.M * a.N) return;
  const int64_t m = e / a.N, n = e % a.N;
  const int lane = threadIdx.x & 63;
  float sum = 0.f;
  for (int64_t k = 8 * lane; k < a.K; k += 512) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(a.W + n * a.ldw + k / 2);
    const int64_t g = k / a.group;
    const float z = a.Z ? (float)a.Z[g * a.ldz + n] : 8.f;
    float part = 0.f;
    for (int i = 0; i < 8; ++i) part = __builtin_fmaf(Elem<Tag>::to_f32(a.A[m * a.lda + k + i]), (float)((w >> (4 * i)) & 15) - z, part);
    sum = __builtin_fmaf(part, Elem<Tag>::to_f32(a.S[g * a.lds + n]), sum);
  }
  sum = wave_sum(sum);
  if (lane == 0) a.C[m * a.ldc + n] = Elem<Tag>::from_f32(sum);
}

}  // namespace

int run_gemm_4bit(const Gemm4bitArgs& a, hipStream_t s, char* name, size_t size) {
  if (a.M > ((int64_t)1 << 40) / a.N) return MLT_ERR_UNSUPPORTED;
  const int64_t wgs = (a.M * a.N + 3) / 4;
  if (!launch_fits(wgs, 256)) return MLT_ERR_UNSUPPORTED;
  auto kern = a.dtype == MLT_BF16 ? gemm_4bit_kernel<bf16_tag> : gemm_4bit_kernel<f16_tag>;
  hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(256), 0, s, a);
  snprintf(name, size, "gemm_4bit_rows");
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

}  // namespace mlt
