// Attention of packed sequences of different lengths, grouped heads, over packed keys or a paged cache (mlt_mha_packed_fwd, mlt_paged_attn_prompt):
// first form. A wavefront owns one (token, query head): 64 keys at a time, a lane's score each, one softmax over them, then the values' rows
// with the lanes along the head's elements.
#include <stdio.h>

#include "attn_rows.h"
#include "mlt_internal.h"

namespace mlt {

namespace {

// the sequence of packed row t: the last b with offsets[b] <= t, if t < offsets[b + 1]; otherwise -1
__device__ __forceinline__ int sequence_of(const int32_t* offsets, int B, int t) {
  int lo = 0, hi = B;                                    // offsets[lo] <= t (if any), offsets[hi] > t (or hi == B)
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (offsets[mid] <= t) lo = mid; else hi = mid;
  }
  return offsets[lo] <= t && t < offsets[lo + 1] ? lo : -1;
}

template <typename Tag, int D>
__global__ __launch_bounds__(256) void prompt_rows_kernel(PromptArgs a, float c) {
  const int64_t w = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
  const int t = (int)(w / a.Hq), q = (int)(w % a.Hq), h = (int)(q / (a.Hq / a.H));
  if (t >= a.T) return;
  const int b = sequence_of(a.q_offsets, (int)a.B, t);
  if (b < 0) return;
  const int64_t n = a.q_offsets[b + 1] - a.q_offsets[b], i = t - a.q_offsets[b];
  const uint16_t* qp = a.Q + t * a.ldq + (int64_t)q * D;
  uint16_t* op = a.O + t * a.ldo + (int64_t)q * D;
  if (a.block_size > 0) {
    const int64_t cap = a.max_blocks * a.block_size;
    int64_t m = a.seq_lens[b];
    m = m < 0 ? 0 : m > cap ? cap : m;
    const int64_t end = m - n + i + 1;
    auto row = [&](int64_t j) {
      int64_t blk = a.block_table[b * a.max_blocks + j / a.block_size];
      blk = blk < 0 ? 0 : blk >= a.num_blocks ? a.num_blocks - 1 : blk;
      return ((blk * a.H + h) * a.block_size + j % a.block_size) * D;
    };
    attend_row<Tag, D>(qp, op, end, a.K, a.V, row, row, c);
  } else {
    int64_t k0 = a.k_offsets[b], k1 = a.k_offsets[b + 1];
    k0 = k0 < 0 ? 0 : k0 > a.Tk ? a.Tk : k0;
    k1 = k1 < k0 ? k0 : k1 > a.Tk ? a.Tk : k1;
    const int64_t end = a.causal ? k1 - k0 - n + i + 1 : k1 - k0;
    attend_row<Tag, D>(qp, op, end, a.K, a.V, [&](int64_t j) { return (k0 + j) * a.ldk + (int64_t)h * D; },
                       [&](int64_t j) { return (k0 + j) * a.ldv + (int64_t)h * D; }, c);
  }
}

}  // namespace

int run_prompt(const PromptArgs& a, hipStream_t s, char* name, size_t size) {
  const int64_t wgs = (a.T * a.Hq + 3) / 4;
  if (!launch_fits(wgs, 256)) return MLT_ERR_UNSUPPORTED;
  const float c = a.scale * 1.4426950408889634f;
  auto kern = a.dtype == MLT_BF16 ? (a.D == 128 ? prompt_rows_kernel<bf16_tag, 128> : prompt_rows_kernel<bf16_tag, 64>)
                                  : (a.D == 128 ? prompt_rows_kernel<f16_tag, 128> : prompt_rows_kernel<f16_tag, 64>);
  hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(256), 0, s, a, c);
  snprintf(name, size, "prompt_rows_d%d", (int)a.D);
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

}  // namespace mlt
