// One query row over keys 0 .. end - 1 by one wavefront (rows of Q and K on 16 bytes): 64 keys at a time, a lane's score each, the running maximum and sum of a softmax, then the
// values' rows with the lanes along the head's elements.
#pragma once

#include "mlt_common.h"

namespace mlt {

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) x = __builtin_fmaxf(x, __shfl_xor(x, s));
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) x += __shfl_xor(x, s);
  return x;
}

// krow(j), vrow(j): key (value) j's row. Ends early where nothing but NaN can come of it.
template <typename Tag, int D, typename KRow, typename VRow>
__device__ __forceinline__ void attend_row(const uint16_t* q, uint16_t* out, int64_t end, KRow krow, VRow vrow, float c) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63;
  float m = -__builtin_inff(), l = 0.f, o[E] = {};
  for (int64_t j0 = 0; j0 < end; j0 += 64) {
    const int64_t j = j0 + lane;
    float s = -__builtin_inff();
    if (j < end) {
      const uint16_t* k = krow(j);
      s = 0.f;
#pragma clang loop unroll(disable)
      for (int d0 = 0; d0 < D; d0 += 32) {
        u32x4 kk[4], qq[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          kk[i] = *reinterpret_cast<const u32x4_mem*>(k + d0 + 8 * i);
          qq[i] = *reinterpret_cast<const u32x4_mem*>(q + d0 + 8 * i);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s = __builtin_fmaf(Elem<Tag>::to_f32((uint16_t)qq[i][e]), Elem<Tag>::to_f32((uint16_t)kk[i][e]), s);
            s = __builtin_fmaf(Elem<Tag>::to_f32((uint16_t)(qq[i][e] >> 16)), Elem<Tag>::to_f32((uint16_t)(kk[i][e] >> 16)), s);
          }
      }
      s *= c;
    }
    const float top = __builtin_fmaxf(m, wave_max(s)), ref = top == -__builtin_inff() ? 0.f : top;
    const float alpha = __builtin_amdgcn_exp2f(m - ref), p = __builtin_amdgcn_exp2f(s - ref);
    l = l * alpha + wave_sum(p);
    m = top;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] *= alpha;
    const int n = end - j0 < 64 ? (int)(end - j0) : 64;
#pragma clang loop unroll(disable)
    for (int i0 = 0; i0 < n; i0 += 8) {                    // eight rows asked for before the first is used
      uint16_t x[8][E];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint16_t* v = vrow(j0 + (i0 + i < n ? i0 + i : n - 1));
#pragma unroll
        for (int e = 0; e < E; ++e) x[i][e] = v[e * 64 + lane];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i0 + i < n) {
          const float w = __shfl(p, i0 + i);
#pragma unroll
          for (int e = 0; e < E; ++e) o[e] = __builtin_fmaf(w, Elem<Tag>::to_f32(x[i][e]), o[e]);
        }
    }
    bool lost = true;
#pragma unroll
    for (int e = 0; e < E; ++e) lost = lost && o[e] != o[e];
    if (__all(lost)) break;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) out[e * 64 + lane] = Elem<Tag>::from_f32(l == 0.f ? o[e] * 0.f : o[e] / l);   // (no key, or none with a weight: scores of -inf)
}

}  // namespace mlt
