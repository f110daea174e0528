// Prompt attention with the keys of a tile of rows split over several workgroups (mlt_mha_packed_fwd, mlt_paged_attn_prompt): few rows and long keys, a short piece of a prompt behind
// a long one, would leave most of the card idle. Parts go to the library's scratch in fp32 (prompt_body); a second kernel joins them.
#include <stdio.h>

#include "prompt_tile.h"

namespace mlt {

namespace {

constexpr int PS_TILES = kPromptPart / PA_BN;

template <typename Tag, int D, bool CAUSAL, bool PAGED>
__global__ __launch_bounds__(PA_NT, 1) void prompt_split_kernel(PromptKernel p, float* part_o, float* part_s) {
  extern __shared__ __align__(16) char smem[];
  PromptSeq seq;
  int b, head, qt;
  if (!prompt_item<PA_BM, PA_NT>(p.items, reinterpret_cast<int*>(smem), seq, b, head, qt)) return;
  seq.q0 = uniform(seq.q0); seq.n = uniform(seq.n); seq.k0 = uniform(seq.k0); seq.m = uniform(seq.m);
  b = uniform(b); head = uniform(head); qt = uniform(qt);
  // equal parts of the tiles that the last row sees, the last ones shorter or without any
  const int rows = seq.n * p.items.G, last = (qt + 1) * PA_BM < rows ? (qt + 1) * PA_BM - 1 : rows - 1;
  const int end = CAUSAL ? seq.m - seq.n + 1 + last / p.items.G : seq.m, tiles = end > 0 ? uniform((end + PA_BN - 1) / PA_BN) : 0;
  const int parts = (int)gridDim.y, part = (int)blockIdx.y;
  int per = (tiles + parts - 1) / parts;
  per = per < PS_TILES ? PS_TILES : per;
  const int t0 = part * per < tiles ? part * per : tiles, n = tiles - t0 < per ? tiles - t0 : per;
  prompt_body<Tag, D, CAUSAL, PAGED, true>(p, seq, b, head, qt, (uint32_t)(uintptr_t)(lptr_t)smem, PromptPart{t0, n, part, parts, part_o, part_s});
}

// A wavefront a row: the parts' results, each with its own reference, on the largest one's. A row whose sequence has no such token is none and stays as it is.
template <typename Tag, int D, bool CAUSAL, bool PAGED>
__global__ __launch_bounds__(256, 8) void prompt_join_kernel(PromptKernel p, const float* __restrict__ part_o, const float* __restrict__ part_s, int parts) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63, G = p.items.G, Hq = p.items.H * G;
  const int64_t q = (int64_t)blockIdx.x * 4 + uniform(threadIdx.x >> 6);
  if (q >= (int64_t)p.items.T * Hq) return;
  const int tok = uniform((int)(q / Hq)), hq = uniform((int)(q % Hq)), head = hq / G;
  PromptSeq seq;
  int b = -1;
  for (int b0 = 0; b0 < p.items.B; b0 += 64) {
    PromptSeq s;
    s.n = 0;
    if (b0 + lane < p.items.B) s.get(p.items, b0 + lane);
    const unsigned long long in = __ballot(s.n > 0 && tok >= s.q0 && tok < s.q0 + s.n);
    if (in) {
      b = b0 + __builtin_ctzll(in);
      break;
    }
  }
  if (b < 0) return;
  b = uniform(b);
  seq.get(p.items, b);
  // lane i: maximum and sum of part i (at most 16); none where the part had no keys (NaN scores leave a maximum of -inf too, but a sum of NaN)
  float mi = -__builtin_inff(), si = 0.f;
  if (lane < parts) {
    mi = part_s[(q * parts + lane) * 2];
    si = part_s[(q * parts + lane) * 2 + 1];
  }
  const unsigned long long some = __ballot(!(mi == -__builtin_inff() && si == 0.f));
  const float M = wave_max(mi), ref = M == -__builtin_inff() ? 0.f : M, wi = __builtin_amdgcn_exp2f(mi - ref);
  const float* so = part_o + q * parts * D + lane * E;
  float acc[E] = {}, S = 0.f;
  for (int i0 = 0; i0 < parts; i0 += 8) {
    float x[8][E];
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) x[k][e] = so[(int64_t)(i0 + k < parts ? i0 + k : i0) * D + e];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float w = __shfl(wi, i0 + k), s = __shfl(si, i0 + k);
      if (some >> (i0 + k) & 1) {
        S += s * w;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += x[k][e] * w;
      }
    }
  }
  const float inv = S == 0.f ? 0.f : 1.f / S;
  uint16_t* out = p.O + (int64_t)tok * p.ldo + (int64_t)hq * D + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) out[e] = Elem<Tag>::from_f32(acc[e] * inv);
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) sum = __builtin_fmaf(acc[e], 0.f, sum);
  if (__any(!(sum == 0.f)) && S - S == 0.f) {             // as at the end of prompt_body
    const int row = (tok - seq.q0) * G + hq % G, last_r = seq.n * G - 1, shift = seq.m - seq.n + 1;
    auto end_of = [&](int r) { return CAUSAL ? shift + (r < last_r ? r : last_r) / G : seq.m; };
    const int there = end_of(row / PA_BM * PA_BM + PA_BM - 1), w_end = end_of(row / 32 * 32 + 31);
    const uint32_t bit = 1u << (row % 32);
    prompt_redo<Tag, D, CAUSAL, PAGED>(p, seq, b, head, row / 32 * 32, bit, S == 0.f ? bit : 0u, (w_end + PA_BN - 1) / PA_BN * PA_BN, there);
  }
}

template <typename Tag, int D, bool CAUSAL, bool PAGED>
int launch_split(const PromptKernel& p, int64_t grid, int parts, float* scratch, hipStream_t s) {
  auto kern = prompt_split_kernel<Tag, D, CAUSAL, PAGED>;
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
  const int64_t rows = (int64_t)p.items.T * p.items.H * p.items.G;
  float* part_s = scratch + rows * parts * D;
  hipLaunchKernelGGL(kern, dim3((unsigned)grid, (unsigned)parts), dim3(PA_NT), PaCfg<D>::SMEM, s, p, scratch, part_s);
  hipLaunchKernelGGL((prompt_join_kernel<Tag, D, CAUSAL, PAGED>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, p, scratch, part_s, parts);
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

template <typename Tag, int D>
int launch_split_t(const PromptKernel& p, int64_t grid, int parts, float* scratch, hipStream_t s) {
  if (p.src.block_table) return launch_split<Tag, D, true, true>(p, grid, parts, scratch, s);
  return p.items.causal ? launch_split<Tag, D, true, false>(p, grid, parts, scratch, s) : launch_split<Tag, D, false, false>(p, grid, parts, scratch, s);
}

}  // namespace

int run_prompt_split(const PromptKernel& p, int dtype, int D, int64_t grid, int parts, float* scratch, hipStream_t s) {
  if (dtype == MLT_BF16) return D == 128 ? launch_split_t<bf16_tag, 128>(p, grid, parts, scratch, s) : launch_split_t<bf16_tag, 64>(p, grid, parts, scratch, s);
  return D == 128 ? launch_split_t<f16_tag, 128>(p, grid, parts, scratch, s) : launch_split_t<f16_tag, 64>(p, grid, parts, scratch, s);
}

}  // namespace mlt
