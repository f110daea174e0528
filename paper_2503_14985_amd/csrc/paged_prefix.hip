// Single-token attention behind a shared prefix (mlt_paged_attn_decode_prefix): first form. A wavefront owns one (sequence, query head) and goes through
// all its keys, those of the prefix by the prefix's table.
#include <stdio.h>

#include "attn_rows.h"
#include "mlt_internal.h"

namespace mlt {

namespace {

template <typename Tag, int D>
__global__ __launch_bounds__(256) void prefix_rows_kernel(PrefixArgs a, float c) {
  const int64_t w = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
  if (w >= a.B * a.Hq) return;
  const int64_t b = w / a.Hq, h = w % a.Hq / (a.Hq / a.H), cap = a.max_blocks * a.block_size;
  int64_t len = a.seq_lens[b];
  len = len < 0 ? 0 : len > cap ? cap : len;
  auto row = [&](int64_t j) {
    int64_t blk = j < a.prefix_len ? a.prefix_table[j / a.block_size] : a.block_table[b * a.max_blocks + j / a.block_size];
    blk = blk < 0 ? 0 : blk >= a.num_blocks ? a.num_blocks - 1 : blk;
    return ((blk * a.H + h) * a.block_size + j % a.block_size) * D;
  };
  attend_row<Tag, D>(a.Q + w * D, a.O + w * D, len, [&](int64_t j) { return a.Kc + row(j); }, [&](int64_t j) { return a.Vc + row(j); }, c);
}

}  // namespace

int64_t paged_prefix_work(const PrefixArgs&) { return 0; }

int run_paged_prefix(const PrefixArgs& a, hipStream_t s, char* name, size_t size) {
  const int64_t wgs = (a.B * a.Hq + 3) / 4;
  if (!launch_fits(wgs, 256)) return MLT_ERR_UNSUPPORTED;
  const float c = a.scale * 1.4426950408889634f;
  auto kern = a.dtype == MLT_BF16 ? (a.D == 128 ? prefix_rows_kernel<bf16_tag, 128> : prefix_rows_kernel<bf16_tag, 64>)
                                  : (a.D == 128 ? prefix_rows_kernel<f16_tag, 128> : prefix_rows_kernel<f16_tag, 64>);
  hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(256), 0, s, a, c);
  snprintf(name, size, "paged_prefix_rows_d%d", (int)a.D);
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

}  // namespace mlt
