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
int launch_prompt(const PromptKernel& p, int64_t grid, hipStream_t s) {
  auto kern = prompt_kernel<Tag, D, CAUSAL, PAGED>;
  static thread_local int configured_dev = -1;          // opt in to > 64 KB LDS once per device
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return MLT_ERR_DEVICE;
  if (configured_dev != dev) {
    if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, PaCfg<D>::SMEM) != hipSuccess) {
      (void)hipGetLastError();
      return MLT_ERR_LAUNCH;
    }
    configured_dev = dev;
  }
  hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(PA_NT), PaCfg<D>::SMEM, s, p);
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

template <typename Tag, int D>
int launch_prompt_t(const PromptKernel& p, int64_t grid, hipStream_t s) {
  if (p.src.block_table) return launch_prompt<Tag, D, true, true>(p, grid, s);
  return p.items.causal ? launch_prompt<Tag, D, true, false>(p, grid, s) : launch_prompt<Tag, D, false, false>(p, grid, s);
}

}  // namespace

int run_prompt(const PromptArgs& a, hipStream_t s, char* name, size_t size) {
  const bool paged = a.block_size > 0, causal = paged || a.causal;
  PromptItems items{(int)a.T, (int)a.Tk, (int)a.B, 0, 0, a.q_offsets, a.k_offsets, a.seq_lens, (int)(a.max_blocks * a.block_size), causal ? 1 : 0, 0, 0, 0, 0, 0, 0.f};
  prompt_teams(items, a.Hq, a.H, PA_BM, device_xcds());
  const int64_t grid = prompt_grid(items, PA_BM);
  // Keys split over several workgroups where there are items for no more than half of the CUs (as far as the host can tell: the lengths are the device's): as many parts as it takes
  // to fill them, none of them without 512 keys of the longest sequence that there may be. One piece of 16 tokens behind 8192 keys (8 items, 16 parts): 150 -> 25 us; 512 behind
  // 32768 (64, 4): 700 -> 249 us; 4 x 16 behind 16384 (32, 8): 285 -> 53 us. With more items than CUs it costs more than it balances (543 tokens of 32 sequences, 320 items,
  // 2 parts: 97 -> 103 us).
  DeviceInfo di;
  const int64_t ncu = device_info(di) && di.ncu > 0 ? di.ncu : 256;
  const int64_t items_guess = ((a.T * items.G + PA_BM - 1) / PA_BM + a.B - 1) * a.H, longest = paged ? items.cap : a.Tk;
  int64_t parts = ncu / items_guess < 16 ? ncu / items_guess : 16;
  if (parts > longest / kPromptPart) parts = longest / kPromptPart;
  float* scratch = nullptr;
  ScratchTurn turn;
  if (parts > 1) scratch = cached_scratch(a.T * a.Hq * parts * (a.D + 2) * 4, s, turn);
  if (!scratch) parts = 1;
  if (!launch_fits(grid * parts, PA_NT)) return MLT_ERR_UNSUPPORTED;
  float c = (a.scale < 0 ? -a.scale : a.scale) * 1.4426950408889634f;   // c > 0 always, as in launch_mha_pp
  if (c < 1e-30f) c = 1e-30f;
  PromptKeys src{a.K, a.V, a.ldk, a.ldv, a.block_table, (int)a.block_size, (int)a.max_blocks, (int)a.num_blocks};
  const PromptKernel p{a.Q, a.O, src, items, a.ldq, a.ldo, c, a.scale < 0 ? 1 : 0};
  if (parts > 1) {
    snprintf(name, size, "prompt_d%d%s%s_256x64_parts%d", (int)a.D, paged ? "_paged" : "", causal ? "_causal" : "", (int)parts);
    return run_prompt_split(p, a.dtype, (int)a.D, grid, (int)parts, scratch, s);
  }
  snprintf(name, size, "prompt_d%d%s%s_256x64", (int)a.D, paged ? "_paged" : "", causal ? "_causal" : "");
  if (a.dtype == MLT_BF16) return a.D == 128 ? launch_prompt_t<bf16_tag, 128>(p, grid, s) : launch_prompt_t<bf16_tag, 64>(p, grid, s);
  return a.D == 128 ? launch_prompt_t<f16_tag, 128>(p, grid, s) : launch_prompt_t<f16_tag, 64>(p, grid, s);
}

}  // namespace mlt
