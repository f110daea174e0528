// Few rows times 4-bit weights with a scale for every group (mlt_gemm_w4): the design of gemm_skinny.hip on packed weights. The cost is reading the weights once, half a byte each.
//
// A workgroup of 8 wavefronts has a share of the columns (rows of the stored weight) in blocks of 16, and all of K or a part of it; the wavefronts split K in pieces of KP. Every wavefront fetches its
// pieces of A and W straight into an LDS ring of its own, several slots ahead, waits for the oldest by count and multiplies: no barrier in the loop. A piece's A stays in
// registers while the blocks of W go by.
//   * Products. W is the first operand of 16x16x32 MFMAs (its 16 rows the columns of C), A the second. A lane's 8 weights of a step are one 32-bit word: nibbles i and i + 4 leave it together
//     (shift, and-or) as the 16-bit numbers 16 + q, which bf16 and fp16 hold exactly in the same way: an exponent of 4 with q as the leading bits of the fraction. That is one
//     operation a weight; subtracting the zero point too would be two and more, and the vector ALU is what the kernel is short of next to memory. Instead the sum over a group is put right:
//       sum a (q - z) = sum a (16 + q) - (16 + z) sum a,
//     the last sum from an MFMA with ones, once for all columns. Both are fp32 over at most 128 products; what cancels between them is a factor of some 6 in size, 2^-20 of the group's
//     sum of |a|: nothing beside the rounding of C. A's elements are put in the order of the nibbles (0 4 1 5 2 6 3 7) when they are read from LDS.
//   * Scales are applied to the fp32 sums of groups. They come in the same stream, a 16-bit number (zero points: 8-bit) for each lane of a load.
//   * With few columns a CU fetches more of A than of W; K is then split over 2, 4 or 8 workgroups (split), whose fp32 partial results the one that comes last at a counter adds in the
//     order of the parts.
// More than 32 rows: gemm_4bit_tile.hip.
//
// 16 x 28672 x 8192 in groups of 128 takes 28.5 us, 4.3 TB/s (one row 24.5, 4.9 TB/s; a copy of the same bytes 26), 1 x 4096 x 4096 5.6, 32 x 28672 x 8192 41. gemm_skinny.hip
// streams as many bytes at 6.6 TB/s, so it is not memory alone: the vector ALU is two thirds busy beside the loads (with weights taken apart by three operations a pair, no constants in registers, it was 33.3 us). 17 to 32 rows
// have twice the products, scales and corrections for a word of weights.
#include <stdio.h>

#include "gemm_4bit.h"
#include "mlt_internal.h"

namespace mlt {

namespace {

constexpr int W4_NW = 8;
constexpr int W4_RING = 19 * 1024 + 512;   // LDS ring of a wavefront: 156 KB in all
constexpr int W4_ROWS = 32;                // rows up to which a wavefront keeps A's piece
constexpr int W4_GB = 8;                   // blocks of 16 columns whose sums are kept at once

// MT: 16-row tiles of A; G: group; KP: k of a piece; ZP: with zero points
template <typename Tag, int MT, int G, int KP, bool ZP>
__global__ __launch_bounds__(W4_NW * 64, 2) void gemm_4bit_kernel(W4 a) {
  typedef typename Elem<Tag>::vec8 V8;
  constexpr int GB = W4_GB, NW = W4_NW, NT = NW * 64;
  constexpr int NS = KP / 32, NG = KP / G, SPG = G / 32;   // steps and groups of a piece, steps of a group
  constexpr int AROW = KP * 2, WROW = KP / 2;              // bytes of a row
  constexpr int ARI = 1024 / AROW, WRI = 1024 / WROW;      // rows of a load
  constexpr int BODY = 4 * AROW, NL = BODY / 1024;         // a slot holds 4 rows of A or 16 of W: loads of it
  constexpr int NSL = (NG * 16 + 63) / 64;                 // loads of a block's scales, of its zero points
  constexpr int SIDE = NSL * 256, SLOT = BODY + SIDE * (ZP ? 2 : 1), SLOTS = W4_RING / SLOT, W_LOADS = NL + NSL * (ZP ? 2 : 1);
  constexpr bool WHOLE = SLOTS >= 5;                       // room for a tile of A and more
  static_assert(BODY == 16 * WROW, "one size for both");
  static_assert(WHOLE || MT == 1, "a tile of A slot by slot: its zeros and sums are those of the last one");
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, g = lane >> 4;
  const int M = a.M, N = a.N, K = a.K;
  const int bid = (int)blockIdx.x, part_id = (int)blockIdx.y;
  const bool split = gridDim.y > 1;
  const int c0 = bid * a.share + (bid < a.rest ? bid : a.rest), c1 = c0 + a.share + (bid < a.rest ? 1 : 0), nblk = (c1 - c0 + 15) / 16;
  const int all = (K + KP - 1) / KP;
  int p0 = 0, p1 = all;
  if (split) {
    const int per = (all + (int)gridDim.y - 1) / (int)gridDim.y;
    p0 = part_id * per;
    p1 = p0 + per < all ? p0 + per : all;
  }
  const int first = p0 + wave, mine = p1 > first ? (p1 - first + NW - 1) / NW : 0;
  // A wavefront begins somewhere in its share and goes round, so that the workgroups are not all at the same place of the rows, which are a power of two apart more often than
  // not: that would be the same few memory channels.
  const int start = mine > 0 ? first + (wave + bid) % mine * NW : first;
  const int last_group = (K - 1) / G;
  const uint32_t ring = (uint32_t)(uintptr_t)(lptr_t)smem + (uint32_t)wave * W4_RING, ring_end = ring + SLOTS * SLOT;
  const int SA = (M + 3) / 4;                              // slots of A

  // A: row 4 i + n of slot i is row n of it, chunk c (8 k) at position c ^ row (low four bits); W: chunk c (32 k) of row n at position c ^ f(n)
  constexpr int ACH = AROW / 16, WCH = WROW / 16;
  auto fw = [](int n) { return WCH == 16 ? n : WCH == 8 ? (n >> 1) & 7 : (n >> 2) & 3; };
  auto side_group = [](int i, int ln) { const int q = (i * 64 + ln) >> 4; return q < NG ? q : NG - 1; };   // a lane's group of the piece (lanes to spare: the last one)
  // per-lane byte offsets of the loads of a slot of W, of its scales and zero points, where all of them are there; and of one of A (its row of the load)
  uint32_t vw[NL], vs[NSL], vz[ZP ? NSL : 1];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int row = i * WRI + lane / WCH;
    vw[i] = (uint32_t)row * (uint32_t)a.ldw + (uint32_t)((lane % WCH) ^ fw(row)) * 16u;
  }
#pragma unroll
  for (int i = 0; i < NSL; ++i) {
    vs[i] = ((uint32_t)side_group(i, lane) * (uint32_t)a.lds + (uint32_t)(lane & 15)) * 2u;
    if (ZP) vz[i] = (uint32_t)side_group(i, lane) * (uint32_t)a.ldz + (uint32_t)(lane & 15);
  }
  const int a_in = lane / ACH;
  const uint32_t a_row = (uint32_t)a_in * (uint32_t)a.lda * 2u, a_chunk = (uint32_t)(((lane % ACH) ^ a_in) * 16);
  // this lane's places in a slot of A (its chunk 4 s + g by XOR, slots begin on 256 bytes) and of W (its word of chunk s)
  const uint32_t a_lane = (uint32_t)((r16 & 3) * AROW + ((g ^ r16) << 4)), w_lane = (uint32_t)(r16 * WROW + (fw(r16) << 4) + 4 * g);
  static_assert(W4_RING % 256 == 0 && SLOT % 256 == 0, "see a_lane");
  uint32_t mask = Nibbles<Tag>::MASK, sixteen = Nibbles<Tag>::SIXTEEN;
  asm volatile("" : "+v"(mask), "+v"(sixteen));

  for (int base = 0; base < nblk; base += GB) {
    const int nb = nblk - base < GB ? nblk - base : GB;
    const int S = SA + nb, T = mine * S;
    f32x4 acc[GB][MT];
#pragma unroll
    for (int b = 0; b < GB; ++b)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) acc[b][mt] = f32x4{0.f, 0.f, 0.f, 0.f};

    // the cursor: the next slot of the stream to fetch, f_s of piece f_p, where its rows begin, and its place
    int f_t = 0, f_s = 0, f_p = start, f_rows = 0, issued = 0, need = 0;
    uint32_t f_slot = ring;
    const uint16_t *f_a = nullptr, *f_sc = nullptr;
    const uint8_t *f_w = nullptr, *f_z = nullptr;
    auto piece_begins = [&]() __attribute__((always_inline)) {
      const int k0 = f_p * KP;
      f_a = a.A + k0;
      f_rows = M;
      f_w = a.W + (int64_t)(c0 + base * 16) * a.ldw + k0 / 2;
      f_sc = a.S + k0 / G * a.lds + c0 + base * 16;
      if (ZP) f_z = a.Z + k0 / G * a.ldz + c0 + base * 16;
    };
    if (T > 0) piece_begins();
    auto fetch = [&]() __attribute__((always_inline)) {
      if (f_t >= T) return;
      const int k0 = f_p * KP;
      const bool tail = k0 + KP > K;                       // chunks past K: the row's first one; they count as zeros
      if (f_s < SA) {
#pragma unroll
        for (int i = 0; i < NL; ++i)
          if (i * ARI < f_rows) {                          // (with several rows a load the last ones may be too many: the first again)
            uint32_t c = a_chunk ^ (uint32_t)(((f_s & 3) * 4 + i * ARI) << 4);
            if (tail && k0 * 2 + (int)c >= K * 2) c = 0;
            load_lds16(f_a + (int64_t)(i * ARI) * a.lda, (ARI > 1 && i * ARI + a_in < f_rows ? a_row : 0u) + c, f_slot + i * 1024u);
            ++issued;
          }
        f_a += 4 * (int64_t)a.lda;
        f_rows -= 4;
      } else {
        if (f_s == SA) f_rows = c1 - (c0 + base * 16);
        if (!tail && f_rows >= 16) {
#pragma unroll
          for (int i = 0; i < NL; ++i) load_lds16_stream(f_w, vw[i], f_slot + i * 1024u);
#pragma unroll
          for (int i = 0; i < NSL; ++i) {
            load_lds_u16(f_sc, vs[i], f_slot + BODY + i * 256u);
            if (ZP) load_lds_u8(f_z, vz[i], f_slot + BODY + SIDE + i * 256u);
          }
        } else {                                           // columns that are not there: the first one's weights, the last one's scales; groups: the last one's
          int ln = lane;
          asm volatile("" : "+v"(ln));
#pragma unroll
          for (int i = 0; i < NL; ++i) {
            const int row = i * WRI + ln / WCH, c = (ln % WCH) ^ fw(row);
            load_lds16_stream(f_w, row < f_rows && k0 + c * 32 < K ? (uint32_t)row * (uint32_t)a.ldw + (uint32_t)c * 16u : 0u, f_slot + i * 1024u);
          }
#pragma unroll
          for (int i = 0; i < NSL; ++i) {
            const int n = (ln & 15) < f_rows ? ln & 15 : f_rows - 1, most = last_group - k0 / G, q = side_group(i, ln) < most ? side_group(i, ln) : most;
            load_lds_u16(f_sc, ((uint32_t)q * (uint32_t)a.lds + n) * 2u, f_slot + BODY + i * 256u);
            if (ZP) load_lds_u8(f_z, (uint32_t)q * (uint32_t)a.ldz + n, f_slot + BODY + SIDE + i * 256u);
          }
        }
        issued += W_LOADS;
        f_w += 16 * (int64_t)a.ldw;
        f_sc += 16;
        if (ZP) f_z += 16;
        f_rows -= 16;
      }
      ++f_t;
      f_slot += SLOT;
      if (f_slot == ring_end) f_slot = ring;
      if (++f_s == S) {
        f_s = 0;
        f_p = f_p + NW < p1 ? f_p + NW : first;
        piece_begins();
      }
    };
#pragma clang loop unroll(disable)
    for (int i = 0; i < SLOTS; ++i) fetch();

    // waits until the next slots, of so many loads, have landed (what was issued after them may be in flight)
    uint32_t slot = ring;
    auto wait = [&](int loads) __attribute__((always_inline)) {
      need += loads;
      int later = issued - need;
#ifdef MLT_DEBUG_BARRIERS
      later = 0;                                           // waits for all of them, so that a count that is too lax shows
#endif
      constexpr int FULL = (SLOTS - 1) * W_LOADS < 63 ? (SLOTS - 1) * W_LOADS : 63;   // (the weights' steady state)
      if (later >= FULL) __builtin_amdgcn_s_waitcnt(wait_imm(FULL, 15));
      else if (later >= FULL * 2 / 3) __builtin_amdgcn_s_waitcnt(wait_imm(FULL * 2 / 3, 15));
      else if (later >= 10) __builtin_amdgcn_s_waitcnt(wait_imm(10, 15));
      else if (later >= 5) __builtin_amdgcn_s_waitcnt(wait_imm(5, 15));
      else if (later >= 2) __builtin_amdgcn_s_waitcnt(wait_imm(2, 15));
      else __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));
      __builtin_amdgcn_sched_barrier(0);
    };
    auto refill = [&](int take) __attribute__((always_inline)) {   // the places of so many slots, which have been read, take the next ones
      __builtin_amdgcn_s_waitcnt(wait_imm(63, 0));
      __builtin_amdgcn_sched_barrier(0);
#pragma clang loop unroll(disable)
      for (int x = 0; x < take; ++x) {
        fetch();
        __builtin_amdgcn_sched_barrier(0);
        slot += SLOT;
        if (slot == ring_end) slot = ring;
      }
    };
    for (int i = 0, piece = start; i < mine; ++i, piece = piece + NW < p1 ? piece + NW : first) {
      const int k0 = piece * KP;
      const bool tail = k0 + KP > K;
      // ---- A: this lane's row r16 of each tile, step s: chunk 4 s + g; and its sums over the groups
      u32x4 af[MT][NS];
      float sa[MT][NG];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int s = 0; s < NS; ++s) af[mt][s] = u32x4{0u, 0u, 0u, 0u};
        const int rows = M - mt * 16 < 16 ? M - mt * 16 : 16;
        if (rows > 0) {
          if (WHOLE) {                                     // each lane reads from its row's slot
            const int take = (rows + 3) / 4;
            wait((rows + ARI - 1) / ARI);
            const uint32_t at = slot + (uint32_t)(r16 < rows ? r16 >> 2 : 0) * (uint32_t)SLOT, from = (at >= ring_end ? at - (uint32_t)(SLOTS * SLOT) : at) + a_lane;
#pragma unroll
            for (int s = 0; s < NS; ++s) af[mt][s] = *(const MLT_LDS u32x4*)(uintptr_t)((from ^ (uint32_t)((s & 3) << 6)) + (uint32_t)((s >> 2) * 256));
            refill(take);
          } else {                                         // slot by slot
            for (int q = 0; q * 4 < rows; ++q) {
              wait((rows - q * 4 < 4 ? rows - q * 4 + ARI - 1 : 4) / ARI);
              if ((r16 >> 2) == q) {
#pragma unroll
                for (int s = 0; s < NS; ++s) af[mt][s] = *(const MLT_LDS u32x4*)(uintptr_t)(((slot + a_lane) ^ (uint32_t)((s & 3) << 6)) + (uint32_t)((s >> 2) * 256));
              }
              refill(1);
            }
          }
        }
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          u32x4 x = af[mt][s];
          if (r16 >= rows || (tail && k0 + 32 * s >= K)) x = u32x4{0u, 0u, 0u, 0u};   // rows that are not there; k past K (whole steps: K is a multiple of 32)
          // the order of the nibbles
          af[mt][s] = u32x4{__builtin_amdgcn_perm(x[2], x[0], 0x05040100u), __builtin_amdgcn_perm(x[2], x[0], 0x07060302u), __builtin_amdgcn_perm(x[3], x[1], 0x05040100u),
                            __builtin_amdgcn_perm(x[3], x[1], 0x07060302u)};
        }
        const uint32_t one = __is_same(Tag, bf16_tag) ? 0x3f803f80u : 0x3c003c00u;
#pragma unroll
        for (int q = 0; q < NG; ++q) {
          f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < SPG; ++s) sum = mfma16(__builtin_bit_cast(V8, u32x4{one, one, one, one}), __builtin_bit_cast(V8, af[mt][q * SPG + s]), sum);
          sa[mt][q] = ZP ? sum[0] : -24.f * sum[0];        // (without zero points: what is to be added)
          asm volatile("" : "+v"(sa[mt][q]));              // (a register of its own: the other three of the four are not to be kept with it)
          __builtin_amdgcn_sched_barrier(0);
        }
      }
#pragma clang loop unroll(disable)
      for (int blk = 0; blk < nb; ++blk) {
        wait(W_LOADS);
        // ---- a block of 16 columns: lane's column r16, step s: word 4 s + g. A group at a time, the next one's numbers read beside this one's products
        uint32_t w[2][SPG];
        u32x4 sc[2], zp[2];                                // scales and zero points of columns 4 g .. 4 g + 3
        f32x4 res[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) res[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
        auto read = [&](int q) __attribute__((always_inline)) {
#pragma unroll
          for (int s = 0; s < SPG; ++s) w[q & 1][s] = *(const MLT_LDS uint32_t*)(uintptr_t)((slot + w_lane) ^ (uint32_t)((q * SPG + s) << 4));
          sc[q & 1] = *(const MLT_LDS u32x4*)(uintptr_t)(slot + BODY + q * 64u + g * 16u);
          if (ZP) zp[q & 1] = *(const MLT_LDS u32x4*)(uintptr_t)(slot + BODY + SIDE + q * 64u + g * 16u);
        };
        read(0);
#pragma unroll
        for (int q = 0; q < NG; ++q) {
          if (q + 1 < NG) read(q + 1);
          f32x4 sum[MT];
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) sum[mt] = ZP ? f32x4{0.f, 0.f, 0.f, 0.f} : f32x4{sa[mt][q], sa[mt][q], sa[mt][q], sa[mt][q]};
#pragma unroll
          for (int s = 0; s < SPG; ++s) {
            const uint32_t x = w[q & 1][s];
            const u32x4 wf = {Nibbles<Tag>::get(x, 0, mask, sixteen), Nibbles<Tag>::get(x, 1, mask, sixteen), Nibbles<Tag>::get(x, 2, mask, sixteen), Nibbles<Tag>::get(x, 3, mask, sixteen)};
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) sum[mt] = mfma16(__builtin_bit_cast(V8, wf), __builtin_bit_cast(V8, af[mt][q * SPG + s]), sum[mt]);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float scale = Elem<Tag>::to_f32((uint16_t)sc[q & 1][r]), off = ZP ? -16.f - (float)zp[q & 1][r] : 0.f;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) res[mt][r] = __builtin_fmaf(ZP ? __builtin_fmaf(off, sa[mt][q], sum[mt][r]) : sum[mt][r], scale, res[mt][r]);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int b = 0; b < GB; ++b)
          if (b == blk) {
            asm volatile("");                              // (jumped over, not selected)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) add4(acc[b][mt], res[mt]);
          }
        refill(1);
      }
    }
    // ---- the wavefronts' sums into their own rings (all their loads have landed), as many blocks at a time as there is room for, then the sums of those.
    // acc register r: column 4 g + r, row r16 of the tile
    float* own = reinterpret_cast<float*>(smem + wave * W4_RING);
    constexpr int FIT = W4_RING / (MT * 1024) < GB ? W4_RING / (MT * 1024) : GB;
#pragma unroll
    for (int b0 = 0; b0 < GB; b0 += FIT) {
      if (b0 >= nb) break;
      if (b0 > 0) __syncthreads();
#pragma unroll
      for (int b = b0; b < b0 + FIT && b < GB; ++b)
        if (b < nb) {
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) *reinterpret_cast<f32x4_mem*>(own + ((b - b0) * MT + mt) * 256 + r16 * 16 + 4 * g) = acc[b][mt];
        }
      __syncthreads();
      const int here = nb - b0 < FIT ? nb - b0 : FIT;
      for (int e = tid; e < here * MT * 256; e += NT) {
        const int t = e >> 8, gr = t % MT * 16 + ((e >> 4) & 15), gc = c0 + (base + b0 + t / MT) * 16 + (e & 15);
        if (gr < M && gc < c1) {
          float sum = 0.f;
#pragma unroll
          for (int w = 0; w < NW; ++w) sum += reinterpret_cast<const float*>(smem)[w * (W4_RING / 4) + e];
          if (split) store_shared(a.part + ((int64_t)part_id * M + gr) * N + gc, sum);
          else a.C[(int64_t)gr * a.ldc + gc] = Elem<Tag>::from_f32(sum);
        }
      }
    }
    if (base + GB < nblk) __syncthreads();
  }
  if (!split) return;

  if (!last_to_arrive(a.counter + bid, gridDim.y, reinterpret_cast<uint32_t*>(smem))) return;
  w4_add_parts<Tag, NT>(a, (int)gridDim.y, 0, M, c0, c1);
}

template <typename Tag, int MT, int G, int KP, bool ZP>
int launch_w4(const W4& a, unsigned nwg, int parts, hipStream_t s) {
  auto kern = gemm_4bit_kernel<Tag, MT, G, KP, ZP>;
  static thread_local int configured_dev = -1;            // opt in to > 64 KB LDS once per device
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return MLT_ERR_DEVICE;
  if (configured_dev != dev) {
    if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, W4_NW * W4_RING) != hipSuccess) {
      (void)hipGetLastError();
      return MLT_ERR_LAUNCH;
    }
    configured_dev = dev;
  }
  hipLaunchKernelGGL(kern, dim3(nwg, (unsigned)parts), dim3(W4_NW * 64), W4_NW * W4_RING, s, a);
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

// 512 k a piece where A's tile and its groups' sums fit the registers (256: 16 x 28672 x 8192 30.9 us instead of 28.3, one row 26.8 instead of 24.7, 1 x 4096 x 4096 7.3 instead of 5.6).
template <typename Tag, int G, bool ZP>
int run_w4_rows(const W4& a, unsigned nwg, int parts, hipStream_t s) {
  if (a.M <= 16) return launch_w4<Tag, 1, G, G == 32 ? 256 : 512, ZP>(a, nwg, parts, s);
  return launch_w4<Tag, 2, G, 256, ZP>(a, nwg, parts, s);
}

template <typename Tag, bool ZP>
int run_w4_t(const W4& a, int group, unsigned nwg, int parts, hipStream_t s) {
  return group == 32 ? run_w4_rows<Tag, 32, ZP>(a, nwg, parts, s) : group == 64 ? run_w4_rows<Tag, 64, ZP>(a, nwg, parts, s) : run_w4_rows<Tag, 128, ZP>(a, nwg, parts, s);
}

__global__ __launch_bounds__(256) void zero_rows_kernel(uint16_t* C, int64_t ldc, int N) {
  for (int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x; n < N; n += (int64_t)gridDim.x * 256) C[(int64_t)blockIdx.y * ldc + n] = 0;
}

}  // namespace

int run_gemm_4bit(const Gemm4bitArgs& g, hipStream_t s, char* name, size_t size) {
  if (g.K == 0) {
    snprintf(name, size, "gemm_4bit_zero");
    const int64_t wide = (g.N + 2047) / 2048, high = ((int64_t)1 << 23) / wide < 65535 ? ((int64_t)1 << 23) / wide : 65535;   // (a launch has 2^32 work-items at most)
    for (int64_t r = 0; r < g.M; r += high) {
      const int64_t n = g.M - r < high ? g.M - r : high;
      hipLaunchKernelGGL(zero_rows_kernel, dim3((unsigned)wide, (unsigned)n), dim3(256), 0, s, g.C + r * g.ldc, g.ldc, (int)g.N);
      if (hipGetLastError() != hipSuccess) return MLT_ERR_LAUNCH;
    }
    return MLT_OK;
  }
  DeviceInfo di;
  const int64_t ncu = device_info(di) && di.ncu > 0 ? di.ncu : 256;
  W4 a{(int)g.M, (int)g.N, (int)g.K, 0, 0, (int)g.lda, (int)g.ldw, g.A, g.W, g.S, g.Z, g.lds, g.ldz, g.C, g.ldc, nullptr, nullptr};
  const bool tile = g.M > W4_ROWS;
  const int64_t rows = g.M <= 16 ? 16 : g.M <= 32 ? 32 : W4T_ROWS, nz = (g.M + rows - 1) / rows, blocks = (g.N + 15) / 16;
  const int64_t wide = (blocks + 15) / 16 * nz * 4 >= ncu ? 16 : 8;   // blocks of a tile (gemm_4bit_tile.hip has the figures)
  int64_t nwg = (blocks + wide - 1) / wide, parts = 1;
  if (tile) {
    // parts of K: rounds of workgroups, each of its chunks and some 4 chunks' time to begin and end, and the kernel that adds them
    const int64_t chunks = (g.K + 127) / 128;
    int64_t best = 0;
    for (int64_t p = 1; p <= 16 && (p == 1 || p * 2 <= chunks); ++p) {
      const int64_t cost = (nwg * nz * p + ncu - 1) / ncu * ((chunks + p - 1) / p + 4) + (p > 1 ? 2 + p / 2 : 0);
      if (p == 1 || cost < best) best = cost, parts = p;
    }
  } else {
    // parts of K until a workgroup reads no more of A than of W (2 rows K / parts against columns K / 2 / parts), as long as each wavefront keeps a piece
    const int64_t kp = rows <= 16 && g.group > 32 ? 512 : 256, pieces = (g.K + kp - 1) / kp;
    while (parts < 8 && rows * 4 * ncu > g.N * parts * 2 && pieces >= 2 * parts * W4_NW) parts *= 2;
  }
  while (parts > 1 && (parts * g.M * g.N * 4 > (int64_t)32 << 20 || (!tile && ncu / parts > kScratchCounters))) parts /= 2;
  ScratchTurn turn;
  if (parts > 1) {
    a.part = cached_scratch(parts * g.M * g.N * 4, s, turn);
    if (a.part) a.counter = scratch_counters(a.part);
  }
  const bool denied = parts > 1 && !a.part;
  if (denied) parts = 1;
  if (tile && denied && g.M <= 2 * W4_ROWS && nwg * nz * 4 <= ncu) {
    // Nothing to split with and tiles for a quarter of the CUs: the rows 32 at a time, by all CUs. Recorded into a graph, as tiles and so: 57 x 4100 x 14336 132 and 90 us,
    // 64 x 8192 x 8192 74 and 47 (three times 32 rows come to the same, four to more).
    for (int64_t r = 0; r < g.M; r += W4_ROWS) {
      Gemm4bitArgs rows32 = g;
      rows32.M = g.M - r < W4_ROWS ? g.M - r : W4_ROWS;
      rows32.A = g.A + r * g.lda;
      rows32.C = g.C + r * g.ldc;
      const int rc = run_gemm_4bit(rows32, s, name, size);
      if (rc != MLT_OK) return rc;
    }
    return MLT_OK;
  }
  if (!tile) {
    nwg = ncu / parts;
    if (nwg > (g.N + 3) / 4) nwg = (g.N + 3) / 4;
  }
  a.share = (int)((tile ? blocks : g.N) / nwg);
  a.rest = (int)((tile ? blocks : g.N) % nwg);
  if (nz > kW4MostTiles || !launch_fits(nwg * parts * nz, 512)) return MLT_ERR_UNSUPPORTED;
  snprintf(name, size, "gemm_4bit_g%d_m%d_parts%d", (int)g.group, (int)rows, (int)parts);
  if (tile) return run_w4_tile(a, g.dtype, (int)g.group, (int)wide, (unsigned)nwg, (int)parts, s);
  if (g.dtype == MLT_BF16) return g.Z ? run_w4_t<bf16_tag, true>(a, (int)g.group, (unsigned)nwg, (int)parts, s) : run_w4_t<bf16_tag, false>(a, (int)g.group, (unsigned)nwg, (int)parts, s);
  return g.Z ? run_w4_t<f16_tag, true>(a, (int)g.group, (unsigned)nwg, (int)parts, s) : run_w4_t<f16_tag, false>(a, (int)g.group, (unsigned)nwg, (int)parts, s);
}

}  // namespace mlt
