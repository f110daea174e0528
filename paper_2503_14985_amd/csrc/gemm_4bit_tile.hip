// mlt_gemm_w4 with more rows than a wavefront can keep: workgroups share A through LDS.
//
// A workgroup of 8 wavefronts has 64 rows and 128 or 256 columns, one or two blocks of 16 columns a wavefront, and all of K or a part of it in chunks of 128. A chunk's A (16 KB) and
// each wavefront's own weights (1 KB a block), scales and zero points go straight into one stage of an LDS ring; one barrier a chunk.
//   * Products as in gemm_4bit.hip: W as the first operand in the form 16 + q, A as the second, a correction by sums of A.
//   * Each chunk's A is put in the order of the nibbles once, in place, by the wavefronts together (two fragments each) while the chunk before is multiplied; the sums of its
//     rows over each step of 32 come along by an MFMA with ones, into LDS.
//   * The correction -(16 + z) s . sum a is itself a product over the four steps: one 16x16x4 fp32 MFMA for each tile and chunk. On the vector ALU it would be 4 operations
//     a tile and group.
// What bounds it is the work around the products, one after the other between two barriers: without them a chunk still takes more than half of its time, most of that A's reads
// from LDS (16 KB a wavefront) and waiting for them. So two blocks a wavefront, which share them, are faster where there are workgroups enough: 64 x 28672 x 8192 66 us, with one
// 76; 128 x 8192 x 8192 43 and 50; but 57 x 4100 x 14336 32 and 30, 48 x 1024 x 1024 12.3 and 9.9. Tiles of 128 rows are slower (128 x 28672 x 8192: 128 us, two of 64 110), and so are
// 16 wavefronts with a block each (as many bytes of A each, 67 us and 43 for the first two).
#include <stdio.h>

#include "gemm_4bit.h"
#include "mlt_internal.h"

namespace mlt {

namespace {

constexpr int W4T_NW = 8, W4T_NT = W4T_NW * 64, W4T_LDS = 160 * 1024;
constexpr int MT = W4T_ROWS / 16;          // tiles of 16 rows

template <typename Tag, int CB, int G, bool ZP>
__global__ __launch_bounds__(W4T_NT, 2) void gemm_4bit_tile_kernel(W4 a) {
  typedef typename Elem<Tag>::vec8 V8;
  constexpr int KC = 128, NG = KC / G, SPG = G / 32;       // k of a chunk, its groups, steps of a group
  constexpr int SLOT = 1024 + 256 * (ZP ? 2 : 1);          // a block's weights, scales and zero points
  constexpr int ATILE = MT * 4096, STAGE = ATILE + W4T_NW * CB * SLOT, SUMS = MT * 256;   // (sums: [step][row], fp32, two buffers)
  constexpr int ST = (W4T_LDS - 2 * SUMS) / STAGE < 6 ? (W4T_LDS - 2 * SUMS) / STAGE : 6;
  static_assert(ST >= 3, "a chunk in use, the next one, one to fetch into");
  constexpr int AL = MT * 4 / W4T_NW;                      // loads of A, fragments of A of a wavefront
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, g = lane >> 4;
  const int m0 = (int)blockIdx.z * MT * 16, M = a.M - m0 < MT * 16 ? a.M - m0 : MT * 16, N = a.N, K = a.K;
  const int bid = (int)blockIdx.x, part_id = (int)blockIdx.y;
  const bool split = gridDim.y > 1;
  const int b0 = bid * a.share + (bid < a.rest ? bid : a.rest), nb = a.share + (bid < a.rest ? 1 : 0);   // blocks of 16 columns, at most 8 CB
  const int c0 = b0 * 16, c1 = c0 + nb * 16 < N ? c0 + nb * 16 : N;
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
  // The wavefront's blocks are wave and wave + 8; a block or column that is not there is the last one again and not written
  const int w_row = lane >> 2, w_chunk = (lane & 3) ^ (w_row >> 2), s_group = w4t_group<G>(g);
  uint32_t vw[CB], vs[CB], vz[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    const int block = (wave + c * W4T_NW < nb ? wave + c * W4T_NW : nb - 1) * 16, w_at = block + w_row < c1 - c0 ? block + w_row : c1 - c0 - 1, s_at = block + r16 < c1 - c0 ? block + r16 : c1 - c0 - 1;
    vw[c] = (uint32_t)w_at * (uint32_t)a.ldw + (uint32_t)w_chunk * 16u;
    vs[c] = ((uint32_t)s_group * (uint32_t)a.lds + (uint32_t)s_at) * 2u;
    vz[c] = ZP ? (uint32_t)s_group * (uint32_t)a.ldz + (uint32_t)s_at : 0u;
  }
  // Chunks in turn from one that differs between the workgroups: rows are a power of two apart more often than not, and all at the same k would be on the same few memory channels.
  int f_t = n > 0 ? (bid + (int)blockIdx.z) % n : 0;
  const uint16_t *f_a, *f_s;
  const uint8_t *f_w, *f_z;
  auto go_to = [&]() __attribute__((always_inline)) {
    f_a = a.A + (int64_t)m0 * a.lda + (int64_t)(t0 + f_t) * KC;
    f_w = a.W + (int64_t)c0 * a.ldw + (int64_t)(t0 + f_t) * (KC / 2);
    f_s = a.S + (int64_t)(t0 + f_t) * NG * a.lds + c0;
    f_z = ZP ? a.Z + (int64_t)(t0 + f_t) * NG * a.ldz + c0 : nullptr;
  };
  go_to();
  uint32_t f_slot = lds;
  // The loads of a chunk in CB + 1 parts, to stand among the products: all wavefronts' loads at once would keep them waiting for the address units
  auto fetch = [&](int part) __attribute__((always_inline)) {
    const int k0 = (t0 + f_t) * KC, left = K - k0;
    const bool tail = left < KC;                           // k past K: A and scales are zeros there, weights the row's first ones
    const uint32_t slot = f_slot, own = slot + ATILE + (uint32_t)wave * (CB * SLOT);
    if (part == 0) {
#pragma unroll
      for (int j = 0; j < AL; ++j) {
        const uint32_t at = slot + (uint32_t)(wave * AL + j) * 1024u;
        if (!tail) load_lds16(f_a, va[j], at);
        else if (((lane & 15) ^ (((wave * AL + j) * 4 + (lane >> 4)) & 15)) * 8 < left) load_lds16(f_a, va[j], at);
        else *(MLT_LDS u32x4*)(uintptr_t)(at + lane * 16u) = u32x4{0u, 0u, 0u, 0u};
      }
      return;
    }
    const int c = part - 1;
    const uint32_t at = own + c * SLOT;
    if (!tail) {
      load_lds16_stream(f_w, vw[c], at);
      load_lds_u16(f_s, vs[c], at + 1024u);
      if (ZP) load_lds_u8(f_z, vz[c], at + 1280u);
    } else {
      load_lds16_stream(f_w, w_chunk * 32 < left ? vw[c] : vw[c] - (uint32_t)w_chunk * 16u, at);
      const bool there = w4t_group_there<G>(k0, g, last_group);
      if (there) load_lds_u16(f_s, vs[c], at + 1024u);
      else *(MLT_LDS uint32_t*)(uintptr_t)(at + 1024u + lane * 4u) = 0u;
      if (ZP) {
        if (there) load_lds_u8(f_z, vz[c], at + 1280u);
        else *(MLT_LDS uint32_t*)(uintptr_t)(at + 1280u + lane * 4u) = 0u;
      }
    }
    if (part < CB) return;
    f_a += KC;
    f_w += KC / 2;
    f_s += NG * a.lds;
    if (ZP) f_z += NG * a.ldz;
    if (++f_t == n) {
      f_t = 0;
      go_to();
    }
    f_slot += STAGE;
    if (f_slot == lds_end) f_slot = lds;
  };
  for (int i = 0; i < ST - 1 && i < n; ++i) {
#pragma unroll
    for (int part = 0; part <= CB; ++part) fetch(part);
  }

  // all but the newest so many chunks have landed
  auto wait = [&](int later) __attribute__((always_inline)) {
    constexpr int L = AL + CB * (ZP ? 3 : 2);
#ifdef MLT_DEBUG_BARRIERS
    later = 0;
#endif
    if (later >= 3 && ST > 5) __builtin_amdgcn_s_waitcnt(wait_imm(3 * L, 15));
    else if (later >= 2 && ST > 4) __builtin_amdgcn_s_waitcnt(wait_imm(2 * L, 15));
    else if (later >= 1 && ST > 3) __builtin_amdgcn_s_waitcnt(wait_imm(L, 15));
    else __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));
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
  u32x4 own_a[AL];
  auto prepare_read = [&](uint32_t slot) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < AL; ++j) {
      const int f = wave * AL + j;
      own_a[j] = *(const MLT_LDS u32x4*)(uintptr_t)(slot + (uint32_t)(f >> 2) * 4096u + (a_lane ^ (uint32_t)((f & 3) << 6)));
    }
  };
  auto prepare = [&](uint32_t slot, uint32_t to) __attribute__((always_inline)) {
    const uint32_t one = __is_same(Tag, bf16_tag) ? 0x3f803f80u : 0x3c003c00u;
#pragma unroll
    for (int j = 0; j < AL; ++j) {
      const int f = wave * AL + j;
      const u32x4 x = own_a[j];
      const u32x4 y = {__builtin_amdgcn_perm(x[2], x[0], 0x05040100u), __builtin_amdgcn_perm(x[2], x[0], 0x07060302u), __builtin_amdgcn_perm(x[3], x[1], 0x05040100u),
                       __builtin_amdgcn_perm(x[3], x[1], 0x07060302u)};
      *(MLT_LDS u32x4*)(uintptr_t)(slot + (uint32_t)(f >> 2) * 4096u + (a_lane ^ (uint32_t)((f & 3) << 6))) = y;
      const f32x4 sum = mfma16(__builtin_bit_cast(V8, u32x4{one, one, one, one}), __builtin_bit_cast(V8, y), f32x4{0.f, 0.f, 0.f, 0.f});
      if (g == 0) *(MLT_LDS float*)(uintptr_t)(to + (uint32_t)((f & 3) * MT * 16 + (f >> 2) * 16 + r16) * 4u) = sum[0];
    }
  };
  const uint32_t w_lane = (uint32_t)(r16 * 64 + ((r16 >> 2) << 4) + 4 * g);
  uint32_t mask = Nibbles<Tag>::MASK, sixteen = Nibbles<Tag>::SIXTEEN;
  asm volatile("" : "+v"(mask), "+v"(sixteen));
  f32x4 res[CB][MT];
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) res[c][mt] = f32x4{0.f, 0.f, 0.f, 0.f};

  uint32_t slot = lds, sum_at = sums;
  if (n > 0) {
    wait(n - 1 < ST - 2 ? n - 1 : ST - 2);
    barrier();
    prepare_read(slot);
    prepare(slot, sum_at);
  }
  for (int i = 0; i < n; ++i) {
    const uint32_t next = slot + STAGE == lds_end ? lds : slot + STAGE, sum_next = sums + sums + SUMS - sum_at;
    if (i + 1 < n) wait(n - i - 2 < ST - 3 ? n - i - 2 : ST - 3);
    barrier();                                             // chunk i is prepared, chunk i + 1 has landed, chunk i - 1 is done with
    const uint32_t own = slot + ATILE + (uint32_t)wave * (CB * SLOT);
    // what the first products need, and the next chunk's fragments, are asked for ahead of the loads
    uint32_t w[CB][4], side_s[CB], side_z[CB];
    float sum_of[MT];
    u32x4 af[2][MT];
    auto read_a = [&](int s) __attribute__((always_inline)) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) af[s & 1][mt] = *(const MLT_LDS u32x4*)(uintptr_t)(slot + (a_lane ^ (uint32_t)(s << 6)) + mt * 4096u);
    };
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int s = 0; s < 4; ++s) w[c][s] = *(const MLT_LDS uint32_t*)(uintptr_t)((own + c * SLOT + w_lane) ^ (uint32_t)(s << 4));
    read_a(0);
    if (i + 1 < n) prepare_read(next);
    const uint32_t side = (uint32_t)((g / SPG) * 16 + r16) * 4u;
#pragma unroll
    for (int c = 0; c < CB; ++c) {
      side_s[c] = *(const MLT_LDS uint32_t*)(uintptr_t)(own + c * SLOT + 1024u + side);
      if (ZP) side_z[c] = *(const MLT_LDS uint32_t*)(uintptr_t)(own + c * SLOT + 1280u + side);
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) sum_of[mt] = *(const MLT_LDS float*)(uintptr_t)(sum_at + (uint32_t)(g * MT * 16 + mt * 16 + r16) * 4u);
    const bool more = i + ST - 1 < n;
#pragma unroll
    for (int q = 0; q < NG; ++q) {
      f32x4 sum[CB][MT];
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) sum[c][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = q * SPG; s < (q + 1) * SPG; ++s) {
        if (s + 1 < 4) read_a(s + 1);
        if (s <= CB && more) fetch(s);
#pragma unroll
        for (int c = 0; c < CB; ++c) {
          const uint32_t x = w[c][s];
          const u32x4 wf = {Nibbles<Tag>::get(x, 0, mask, sixteen), Nibbles<Tag>::get(x, 1, mask, sixteen), Nibbles<Tag>::get(x, 2, mask, sixteen), Nibbles<Tag>::get(x, 3, mask, sixteen)};
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) sum[c][mt] = mfma16(__builtin_bit_cast(V8, wf), __builtin_bit_cast(V8, af[s & 1][mt]), sum[c][mt]);
        }
      }
      if (q == 0) {  // the correction: step g of column r16 against step g of row r16
#pragma unroll
        for (int c = 0; c < CB; ++c) {
          const float scale = Elem<Tag>::to_f32((uint16_t)side_s[c]), off = scale * (ZP ? -16.f - (float)side_z[c] : -24.f);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) res[c][mt] = __builtin_amdgcn_mfma_f32_16x16x4f32(off, sum_of[mt], res[c][mt], 0, 0, 0);
        }
      }
#pragma unroll
      for (int c = 0; c < CB; ++c) {
        const u32x4 sc = *(const MLT_LDS u32x4*)(uintptr_t)(own + c * SLOT + 1024u + q * 64u + g * 16u);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float scale = Elem<Tag>::to_f32((uint16_t)sc[r]);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) res[c][mt][r] = __builtin_fmaf(sum[c][mt][r], scale, res[c][mt][r]);
        }
      }
    }
    if (i + 1 < n) prepare(next, sum_next);
    slot = next;
    sum_at = sum_next;
  }
  __syncthreads();
  // res register r: column 4 g + r, row r16 of the tile. Through LDS (rows of 128 and 4 to keep them off each other's banks), so that rows are stored in order
  constexpr int ROW = 132;
  float* out = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    if (c > 0) __syncthreads();
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) *reinterpret_cast<f32x4_mem*>(out + (mt * 16 + r16) * ROW + wave * 16 + 4 * g) = res[c][mt];
    __syncthreads();
    for (int e = tid; e < M * 128; e += W4T_NT) {
      const int row = e >> 7, col = c * 128 + (e & 127);
      if (c0 + col < c1) {
        const float v = out[row * ROW + (e & 127)];
        if (split) a.part[((int64_t)part_id * a.M + m0 + row) * N + c0 + col] = v;
        else a.C[(int64_t)(m0 + row) * a.ldc + c0 + col] = Elem<Tag>::from_f32(v);
      }
    }
  }
}

// The sums of the parts, in their order. A kernel of its own (4 us for 7 parts of 57 x 4100): the last workgroup of some columns to end would have to read all their parts alone, 16 us of
// 44 with 13 parts of those, where this leaves 32.
template <typename Tag> __global__ __launch_bounds__(256) void gemm_4bit_add_kernel(W4 a, int parts) {
  const int64_t size = (int64_t)a.M * a.N, e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= size) return;
  float sum = 0.f;
  for (int p0 = 0; p0 < parts; p0 += 8) {
    float v[8];
#pragma unroll
    for (int p = 0; p < 8; ++p) v[p] = a.part[(p0 + p < parts ? p0 + p : p0) * size + e];
#pragma unroll
    for (int p = 0; p < 8; ++p) sum += p0 + p < parts ? v[p] : 0.f;
  }
  a.C[e / a.N * a.ldc + e % a.N] = Elem<Tag>::from_f32(sum);
}

template <typename Tag, int CB, int G, bool ZP>
int launch_tile(const W4& a, unsigned nwg, int parts, hipStream_t s) {
  auto kern = gemm_4bit_tile_kernel<Tag, CB, G, ZP>;
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
  if (parts > 1) hipLaunchKernelGGL(gemm_4bit_add_kernel<Tag>, dim3((unsigned)(((int64_t)a.M * a.N + 255) / 256)), dim3(256), 0, s, a, parts);
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

template <typename Tag, int G, bool ZP>
int launch_cols(const W4& a, int blocks, unsigned nwg, int parts, hipStream_t s) {
  return blocks == 8 ? launch_tile<Tag, 1, G, ZP>(a, nwg, parts, s) : launch_tile<Tag, 2, G, ZP>(a, nwg, parts, s);
}
template <typename Tag, bool ZP>
int launch_group(const W4& a, int group, int blocks, unsigned nwg, int parts, hipStream_t s) {
  return group == 32 ? launch_cols<Tag, 32, ZP>(a, blocks, nwg, parts, s)
                     : group == 64 ? launch_cols<Tag, 64, ZP>(a, blocks, nwg, parts, s) : launch_cols<Tag, 128, ZP>(a, blocks, nwg, parts, s);
}

}  // namespace

int run_w4_tile(const W4& a, int dtype, int group, int blocks, unsigned nwg, int parts, hipStream_t s) {
  if (dtype == MLT_BF16) return a.Z ? launch_group<bf16_tag, true>(a, group, blocks, nwg, parts, s) : launch_group<bf16_tag, false>(a, group, blocks, nwg, parts, s);
  return a.Z ? launch_group<f16_tag, true>(a, group, blocks, nwg, parts, s) : launch_group<f16_tag, false>(a, group, blocks, nwg, parts, s);
}

}  // namespace mlt
