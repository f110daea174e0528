// mlt_gemm_w4 with more rows than a wavefront can keep: workgroups share A through LDS.
//
// A workgroup of 8 wavefronts has MT tiles of 16 rows and 128 columns, one block of 16 columns a wavefront, and all of K or a part of it in chunks of 128. A chunk's A (MT x 4 KB) and
// each wavefront's own weights (1 KB), scales and zero points go straight into one stage of an LDS ring; one barrier a chunk.
//   * Products as in gemm_4bit.hip: W as the first operand in the form 16 + q, A as the second, a correction by sums of A.
//   * Each chunk's A is put in the order of the nibbles once, in place, by the wavefronts together (MT / 2 fragments each) while the chunk before is multiplied; the sums of its
//     rows over each step of 32 come along by an MFMA with ones, into LDS.
//   * The correction -(16 + z) s . sum a is itself a product over the four steps: one 16x16x4 fp32 MFMA for each tile and chunk. On the vector ALU it would be 4 operations
//     a tile and group.
#include <stdio.h>

#include "gemm_4bit.h"
#include "mlt_internal.h"

namespace mlt {

namespace {

constexpr int W4T_NW = 8, W4T_NT = W4T_NW * 64, W4T_LDS = 160 * 1024;

template <typename Tag, int MT, int G, bool ZP>
__global__ __launch_bounds__(W4T_NT, 2) void gemm_4bit_tile_kernel(W4 a) {
  typedef typename Elem<Tag>::vec8 V8;
  constexpr int KC = 128, NG = KC / G, SPG = G / 32;       // k of a chunk, its groups, steps of a group
  constexpr int SLOT = 1024 + 256 * (ZP ? 2 : 1);          // a wavefront's weights, scales and zero points
  constexpr int ATILE = MT * 4096, STAGE = ATILE + W4T_NW * SLOT, SUMS = MT * 256;   // (sums: [step][row], fp32, two buffers)
  constexpr int ST = (W4T_LDS - 2 * SUMS) / STAGE < 6 ? (W4T_LDS - 2 * SUMS) / STAGE : 6;
  static_assert(ST >= 3, "a chunk in use, the next one, one to fetch into");
  constexpr int AL = MT >= 2 ? MT / 2 : 1;                 // loads of A, fragments of A of a wavefront (MT = 1: of the first four)
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, g = lane >> 4;
  const bool a_mine = MT >= 2 || wave < 4;
  const int m0 = (int)blockIdx.z * MT * 16, M = a.M - m0 < MT * 16 ? a.M - m0 : MT * 16, N = a.N, K = a.K;
  const int bid = (int)blockIdx.x, part_id = (int)blockIdx.y;
  const bool split = gridDim.y > 1;
  const int b0 = bid * a.share + (bid < a.rest ? bid : a.rest), nb = a.share + (bid < a.rest ? 1 : 0);   // blocks of 16 columns, at most 8
  const int c0 = b0 * 16, c1 = c0 + nb * 16 < N ? c0 + nb * 16 : N;
  const int cw = c0 + (wave < nb ? wave : nb - 1) * 16, cols = N - cw < 16 ? N - cw : 16;                  // (a wavefront without a block: the last one's, not written)
  const int all = (K + KC - 1) / KC, per = (all + (int)gridDim.y - 1) / (int)gridDim.y;
  const int t0 = part_id * per, n = t0 + per < all ? per : all - t0 > 0 ? all - t0 : 0;
  const int last_group = (K - 1) / G;
  const uint32_t lds = (uint32_t)(uintptr_t)(lptr_t)smem, lds_end = lds + ST * STAGE, sums = lds_end;

  // A: row r at 256 r of the tile, its chunk c (8 k) at position c ^ r (low four bits). W: chunk c (32 k) of row n of the block at position c ^ (n >> 2)
  uint32_t va[AL];
#pragma unroll
  for (int j = 0; j < AL; ++j) {
    const int row = (wave * AL + j) * 4 + (lane >> 4);
    va[j] = (uint32_t)(row < M ? row : M - 1) * (uint32_t)a.lda * 2u + (uint32_t)((lane & 15) ^ (row & 15)) * 16u;
  }
  const int w_row = lane >> 2, w_chunk = (lane & 3) ^ (w_row >> 2);
  const uint32_t vw = (uint32_t)(w_row < cols ? w_row : cols - 1) * (uint32_t)a.ldw + (uint32_t)w_chunk * 16u;
  const int s_group = g < NG ? g : NG - 1, s_col = r16 < cols ? r16 : cols - 1;
  const uint32_t vs = ((uint32_t)s_group * (uint32_t)a.lds + (uint32_t)s_col) * 2u, vz = ZP ? (uint32_t)s_group * (uint32_t)a.ldz + (uint32_t)s_col : 0u;
  const uint16_t* f_a = a.A + (int64_t)m0 * a.lda + (int64_t)t0 * KC;
  const uint8_t* f_w = a.W + (int64_t)cw * a.ldw + (int64_t)t0 * (KC / 2);
  const uint16_t* f_s = a.S + (int64_t)t0 * NG * a.lds + cw;
  const uint8_t* f_z = ZP ? a.Z + (int64_t)t0 * NG * a.ldz + cw : nullptr;
  int f_t = 0;
  uint32_t f_slot = lds;
  auto fetch = [&]() __attribute__((always_inline)) {
    const int k0 = (t0 + f_t) * KC;
    const uint32_t slot = f_slot, own = slot + ATILE + (uint32_t)wave * SLOT;
    if (k0 + KC <= K) {
      if (a_mine) {
#pragma unroll
        for (int j = 0; j < AL; ++j) load_lds16(f_a, va[j], slot + (uint32_t)(wave * AL + j) * 1024u);
      }
      load_lds16_stream(f_w, vw, own);
      load_lds_u16(f_s, vs, own + 1024u);
      if (ZP) load_lds_u8(f_z, vz, own + 1280u);
    } else {                                               // k past K: A and scales are zeros there, weights the row's first ones
      const int left = K - k0;
      if (a_mine) {
#pragma unroll
        for (int j = 0; j < AL; ++j) {
          const int row = (wave * AL + j) * 4 + (lane >> 4);
          const uint32_t at = slot + (uint32_t)(wave * AL + j) * 1024u;
          if (((lane & 15) ^ (row & 15)) * 8 < left) load_lds16(f_a, va[j], at);
          else *(MLT_LDS u32x4*)(uintptr_t)(at + lane * 16u) = u32x4{0u, 0u, 0u, 0u};
        }
      }
      load_lds16_stream(f_w, w_chunk * 32 < left ? vw : vw - (uint32_t)w_chunk * 16u, own);
      const bool there = k0 / G + g <= last_group || g >= NG;
      if (there) load_lds_u16(f_s, vs, own + 1024u);
      else *(MLT_LDS uint32_t*)(uintptr_t)(own + 1024u + lane * 4u) = 0u;
      if (ZP) {
        if (there) load_lds_u8(f_z, vz, own + 1280u);
        else *(MLT_LDS uint32_t*)(uintptr_t)(own + 1280u + lane * 4u) = 0u;
      }
    }
    f_a += KC;
    f_w += KC / 2;
    f_s += NG * a.lds;
    if (ZP) f_z += NG * a.ldz;
    ++f_t;
    f_slot += STAGE;
    if (f_slot == lds_end) f_slot = lds;
  };
  for (int i = 0; i < ST - 1 && i < n; ++i) fetch();

  // all but the newest so many chunks have landed
  auto wait = [&](int later) __attribute__((always_inline)) {
    constexpr int W = 2 + (ZP ? 1 : 0), L = W + AL;
#ifdef MLT_DEBUG_BARRIERS
    later = 0;
#endif
    if (MT >= 2 || a_mine) {
      if (later >= 3 && ST > 5) __builtin_amdgcn_s_waitcnt(wait_imm(3 * L, 15));
      else if (later >= 2 && ST > 4) __builtin_amdgcn_s_waitcnt(wait_imm(2 * L, 15));
      else if (later >= 1 && ST > 3) __builtin_amdgcn_s_waitcnt(wait_imm(L, 15));
      else __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));
    } else {
      if (later >= 3 && ST > 5) __builtin_amdgcn_s_waitcnt(wait_imm(3 * W, 15));
      else if (later >= 2 && ST > 4) __builtin_amdgcn_s_waitcnt(wait_imm(2 * W, 15));
      else if (later >= 1 && ST > 3) __builtin_amdgcn_s_waitcnt(wait_imm(W, 15));
      else __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto barrier = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(wait_imm(63, 0));
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };
  // a chunk that has landed: its fragments of this wavefront (tile f / 4, step f % 4) into the order of the nibbles (0 4 1 5 2 6 3 7), their rows' sums to [step][row]
  const uint32_t a_lane = (uint32_t)(r16 * 256 + ((g ^ r16) << 4));
  auto prepare = [&](uint32_t slot, uint32_t to) __attribute__((always_inline)) {
    if (!a_mine) return;
    const uint32_t one = __is_same(Tag, bf16_tag) ? 0x3f803f80u : 0x3c003c00u;
#pragma unroll
    for (int j = 0; j < AL; ++j) {
      const int f = wave * AL + j;
      const uint32_t at = slot + (uint32_t)(f >> 2) * 4096u + (a_lane ^ (uint32_t)((f & 3) << 6));
      const u32x4 x = *(const MLT_LDS u32x4*)(uintptr_t)at;
      const u32x4 y = {__builtin_amdgcn_perm(x[2], x[0], 0x05040100u), __builtin_amdgcn_perm(x[2], x[0], 0x07060302u), __builtin_amdgcn_perm(x[3], x[1], 0x05040100u),
                       __builtin_amdgcn_perm(x[3], x[1], 0x07060302u)};
      *(MLT_LDS u32x4*)(uintptr_t)at = y;
      const f32x4 sum = mfma16(__builtin_bit_cast(V8, u32x4{one, one, one, one}), __builtin_bit_cast(V8, y), f32x4{0.f, 0.f, 0.f, 0.f});
      if (g == 0) *(MLT_LDS float*)(uintptr_t)(to + (uint32_t)((f & 3) * MT * 16 + (f >> 2) * 16 + r16) * 4u) = sum[0];
    }
  };
  const uint32_t w_lane = (uint32_t)(r16 * 64 + ((r16 >> 2) << 4) + 4 * g);
  uint32_t mask = Nibbles<Tag>::MASK, sixteen = Nibbles<Tag>::SIXTEEN;
  asm volatile("" : "+v"(mask), "+v"(sixteen));
  f32x4 res[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) res[mt] = f32x4{0.f, 0.f, 0.f, 0.f};

  uint32_t slot = lds, sum_at = sums;
  if (n > 0) {
    wait(n - 1 < ST - 2 ? n - 1 : ST - 2);
    barrier();
    prepare(slot, sum_at);
  }
  for (int i = 0; i < n; ++i) {
    const uint32_t next = slot + STAGE == lds_end ? lds : slot + STAGE, sum_next = sums + sums + SUMS - sum_at;
    if (i + 1 < n) wait(n - i - 2 < ST - 3 ? n - i - 2 : ST - 3);
    barrier();                                             // chunk i is prepared, chunk i + 1 has landed, chunk i - 1 is done with
    if (i + ST - 1 < n) fetch();
    if (i + 1 < n) prepare(next, sum_next);
    const uint32_t own = slot + ATILE + (uint32_t)wave * SLOT;
    {  // the correction: step g of column r16 against step g of row r16
      const uint32_t side = (uint32_t)((g / SPG) * 16 + r16) * 4u;
      const float scale = Elem<Tag>::to_f32((uint16_t) * (const MLT_LDS uint32_t*)(uintptr_t)(own + 1024u + side));
      const float off = scale * (ZP ? -16.f - (float)*(const MLT_LDS uint32_t*)(uintptr_t)(own + 1280u + side) : -24.f);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        res[mt] = __builtin_amdgcn_mfma_f32_16x16x4f32(off, *(const MLT_LDS float*)(uintptr_t)(sum_at + (uint32_t)(g * MT * 16 + mt * 16 + r16) * 4u), res[mt], 0, 0, 0);
    }
#pragma unroll
    for (int q = 0; q < NG; ++q) {
      f32x4 sum[MT];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) sum[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = q * SPG; s < (q + 1) * SPG; ++s) {
        const uint32_t x = *(const MLT_LDS uint32_t*)(uintptr_t)((own + w_lane) ^ (uint32_t)(s << 4));
        const u32x4 wf = {Nibbles<Tag>::get(x, 0, mask, sixteen), Nibbles<Tag>::get(x, 1, mask, sixteen), Nibbles<Tag>::get(x, 2, mask, sixteen), Nibbles<Tag>::get(x, 3, mask, sixteen)};
        const uint32_t at = slot + (a_lane ^ (uint32_t)(s << 6));
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          sum[mt] = mfma16(__builtin_bit_cast(V8, wf), __builtin_bit_cast(V8, *(const MLT_LDS u32x4*)(uintptr_t)(at + mt * 4096u)), sum[mt]);
      }
      const u32x4 sc = *(const MLT_LDS u32x4*)(uintptr_t)(own + 1024u + q * 64u + g * 16u);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float scale = Elem<Tag>::to_f32((uint16_t)sc[r]);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) res[mt][r] = __builtin_fmaf(sum[mt][r], scale, res[mt][r]);
      }
    }
    slot = next;
    sum_at = sum_next;
  }
  __syncthreads();
  // res register r: column 4 g + r, row r16 of the tile. Through LDS (rows of 128 and 4 to keep them off each other's banks), so that rows are stored in order
  constexpr int ROW = 132;
  float* out = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) *reinterpret_cast<f32x4_mem*>(out + (mt * 16 + r16) * ROW + wave * 16 + 4 * g) = res[mt];
  __syncthreads();
  for (int e = tid; e < M * 128; e += W4T_NT) {
    const int row = e >> 7, col = e & 127;
    if (c0 + col < c1) {
      const float v = out[row * ROW + col];
      if (split) store_shared(a.part + ((int64_t)part_id * a.M + m0 + row) * N + c0 + col, v);
      else a.C[(int64_t)(m0 + row) * a.ldc + c0 + col] = Elem<Tag>::from_f32(v);
    }
  }
  if (!split) return;
  if (!last_to_arrive(a.counter + bid * (int)gridDim.z + (int)blockIdx.z, gridDim.y, reinterpret_cast<uint32_t*>(smem + W4T_LDS - 16))) return;
  w4_add_parts<Tag, W4T_NT>(a, (int)gridDim.y, m0, M, c0, c1);
}

template <typename Tag, int MT, int G, bool ZP>
int launch_tile(const W4& a, unsigned nwg, int parts, hipStream_t s) {
  auto kern = gemm_4bit_tile_kernel<Tag, MT, G, ZP>;
  static thread_local int configured_dev = -1;            // opt in to > 64 KB LDS once per device
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return MLT_ERR_DEVICE;
  if (configured_dev != dev) {
    if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, W4T_LDS) != hipSuccess) {
      (void)hipGetLastError();
      return MLT_ERR_LAUNCH;
    }
    configured_dev = dev;
  }
  hipLaunchKernelGGL(kern, dim3(nwg, (unsigned)parts, (unsigned)((a.M + MT * 16 - 1) / (MT * 16))), dim3(W4T_NT), W4T_LDS, s, a);
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

template <typename Tag, int G, bool ZP>
int launch_rows(const W4& a, int rows, unsigned nwg, int parts, hipStream_t s) {
  return rows <= 32 ? launch_tile<Tag, 2, G, ZP>(a, nwg, parts, s) : rows <= 64 ? launch_tile<Tag, 4, G, ZP>(a, nwg, parts, s) : launch_tile<Tag, 8, G, ZP>(a, nwg, parts, s);
}
template <typename Tag, bool ZP>
int launch_group(const W4& a, int group, int rows, unsigned nwg, int parts, hipStream_t s) {
  return group == 32 ? launch_rows<Tag, 32, ZP>(a, rows, nwg, parts, s)
                     : group == 64 ? launch_rows<Tag, 64, ZP>(a, rows, nwg, parts, s) : launch_rows<Tag, 128, ZP>(a, rows, nwg, parts, s);
}

}  // namespace

int run_w4_tile(const W4& a, int dtype, int group, int rows, unsigned nwg, int parts, hipStream_t s) {
  if (dtype == MLT_BF16) return a.Z ? launch_group<bf16_tag, true>(a, group, rows, nwg, parts, s) : launch_group<bf16_tag, false>(a, group, rows, nwg, parts, s);
  return a.Z ? launch_group<f16_tag, true>(a, group, rows, nwg, parts, s) : launch_group<f16_tag, false>(a, group, rows, nwg, parts, s);
}

}  // namespace mlt
