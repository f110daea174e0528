// Attention of packed sequences of different lengths, grouped heads, over packed keys or a paged cache (mlt_mha_packed_fwd, mlt_paged_attn_prompt).
// What a workgroup does with its item, and which one it takes, is in prompt_tile.h.
#include <stdio.h>

#include "prompt_tile.h"

namespace mlt {

namespace {

template <typename Tag, int D, bool CAUSAL, bool PAGED>
__global__ __launch_bounds__(PA_NT, D == 64 ? 4 : 1) void prompt_kernel(PromptKernel p) {
  extern __shared__ __align__(16) char smem[];
  PromptSeq seq;
  int b, head, qt;
  if (!prompt_item<PA_BM, PA_NT>(p.items, reinterpret_cast<int*>(smem), seq, b, head, qt)) return;
  seq.q0 = uniform(seq.q0); seq.n = uniform(seq.n); seq.k0 = uniform(seq.k0); seq.m = uniform(seq.m);
  b = uniform(b); head = uniform(head); qt = uniform(qt);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lptr_t)smem;
  prompt_body<Tag, D, CAUSAL, PAGED, false>(p, seq, b, head, qt, lds0, PromptPart{});
}

template <typename Tag, int D, bool CAUSAL, bool PAGED>
int launch_prompt(const PromptArgs& a, hipStream_t s) {
  typedef PaCfg<D> L;
  auto kern = prompt_kernel<Tag, D, CAUSAL, PAGED>;
  PromptItems items{(int)a.T, (int)a.Tk, (int)a.B, 0, 0, a.q_offsets, a.k_offsets, a.seq_lens, (int)(a.max_blocks * a.block_size), CAUSAL ? 1 : 0, 0, 0, 0, 0, 0, 0.f};
  prompt_teams(items, a.Hq, a.H, PA_BM, device_xcds());
  const int64_t grid = prompt_grid(items, PA_BM);
  if (!launch_fits(grid, PA_NT)) return MLT_ERR_UNSUPPORTED;
  static thread_local int configured_dev = -1;          // opt in to > 64 KB LDS once per device
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return MLT_ERR_DEVICE;
  if (configured_dev != dev) {
    if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, L::SMEM) != hipSuccess) {
      (void)hipGetLastError();
      return MLT_ERR_LAUNCH;
    }
    configured_dev = dev;
  }
  float c = (a.scale < 0 ? -a.scale : a.scale) * 1.4426950408889634f;   // c > 0 always, as in launch_mha_pp
  if (c < 1e-30f) c = 1e-30f;
  PromptKeys src{a.K, a.V, a.ldk, a.ldv, a.block_table, (int)a.block_size, (int)a.max_blocks, (int)a.num_blocks};
  hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(PA_NT), L::SMEM, s, PromptKernel{a.Q, a.O, src, items, a.ldq, a.ldo, c, a.scale < 0 ? 1 : 0});
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

template <typename Tag, int D>
int run_prompt_t(const PromptArgs& a, hipStream_t s) {
  if (a.block_size > 0) return launch_prompt<Tag, D, true, true>(a, s);
  return a.causal ? launch_prompt<Tag, D, true, false>(a, s) : launch_prompt<Tag, D, false, false>(a, s);
}

}  // namespace

int run_prompt(const PromptArgs& a, hipStream_t s, char* name, size_t size) {
  snprintf(name, size, "prompt_d%d%s%s_256x64", (int)a.D, a.block_size > 0 ? "_paged" : "", a.causal ? "_causal" : "");
  if (a.dtype == MLT_BF16) return a.D == 128 ? run_prompt_t<bf16_tag, 128>(a, s) : run_prompt_t<bf16_tag, 64>(a, s);
  return a.D == 128 ? run_prompt_t<f16_tag, 128>(a, s) : run_prompt_t<f16_tag, 64>(a, s);
}

}  // namespace mlt
