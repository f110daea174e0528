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
// More than 64 rows are tiles of 64, which read the weights once each.
#include <stdio.h>

#include "fp8.h"
#include "mlt_internal.h"

namespace mlt {

namespace {

constexpr int W4_NW = 8, W4_NT = W4_NW * 64;
constexpr int W4_RING = 19 * 1024 + 512;   // LDS ring of a wavefront: 156 KB in all
constexpr int W4_ROWS = 64;                // rows of C of a workgroup

// a 16-bit (8-bit) number for each lane (uniform base + per-lane byte offset), as a dword to lds_addr + 4 * lane
__device__ __forceinline__ void load_lds_u16(const void* base, uint32_t voff, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ushort %1, %2" : : "s"(lds_addr), "v"(voff), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void load_lds_u8(const void* base, uint32_t voff, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ubyte %1, %2" : : "s"(lds_addr), "v"(voff), "s"(base) : "memory", "m0");
}

// 16 + q of nibbles i and i + 4
template <typename Tag> __device__ __forceinline__ uint32_t nibbles(uint32_t w, int i) {
  if constexpr (__is_same(Tag, bf16_tag)) {
    const uint32_t x = i == 0 ? w << 3 : w >> (4 * i - 3);
    return (x & 0x00780078u) | 0x41804180u;
  } else {
    const uint32_t x = i < 2 ? w << (6 - 4 * i) : w >> (4 * i - 6);
    return (x & 0x03c003c0u) | 0x4c004c00u;
  }
}

struct W4 {
  int M, N, K, share, rest, lda, ldw;
  const uint16_t* A;
  const uint8_t* W;
  const uint16_t* S;
  const uint8_t* Z;
  int64_t lds, ldz;                            // (below 2^26)
  uint16_t* C;
  int64_t ldc;
  float* part;
  uint32_t* counter;
};

// MT: 16-row tiles of A; G: group; KP: k of a piece; GB: blocks of columns in a group of blocks, at most
template <typename Tag, int MT, int G, int KP, int GB>
__global__ __launch_bounds__(W4_NT, 2) void gemm_4bit_kernel(W4 a) {
  typedef typename Elem<Tag>::vec8 V8;
  constexpr int NS = KP / 32, NG = KP / G, SPG = G / 32;   // steps and groups of a piece, steps of a group
  constexpr int AROW = KP * 2, WROW = KP / 2;              // bytes of a row
  constexpr int ARI = 1024 / AROW, WRI = 1024 / WROW;      // rows of a load: 1 or 2, 4 or 8
  constexpr int BODY = 4 * AROW, NL = BODY / 1024;         // a slot holds 4 rows of A or 16 of W: loads of it
  constexpr int NSL = (NG * 16 + 63) / 64;                 // loads of a block's scales, of its zero points
  constexpr int SIDE = NSL * 256;
  static_assert(BODY == 16 * WROW, "one size for both");
  constexpr bool WHOLE = KP == 256;
  static_assert(!WHOLE || W4_RING / (BODY + 2 * SIDE) >= 4, "room for a tile of A");
  static_assert(WHOLE || MT == 1, "a tile of A slot by slot: its zeros and sums are those of the last one");
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, g = lane >> 4;
  const int m0 = (int)blockIdx.z * W4_ROWS, M = a.M - m0 < W4_ROWS ? a.M - m0 : W4_ROWS, N = a.N, K = a.K;
  const uint16_t* const A = a.A + (int64_t)m0 * a.lda;
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
  const int first = p0 + wave, mine = p1 > first ? (p1 - first + W4_NW - 1) / W4_NW : 0;
  const int last_group = (K - 1) / G;
  const int slot_bytes = BODY + SIDE * (a.Z ? 2 : 1), slots = W4_RING / slot_bytes;
  const uint32_t ring = (uint32_t)(uintptr_t)(lptr_t)smem + (uint32_t)wave * W4_RING, ring_end = ring + slots * slot_bytes;
  const int SA = (M + 3) / 4;                              // slots of A

  // A: row 4 i + n of slot i is row n of it, chunk c (8 k) at position c ^ row (low four bits); W: chunk c (32 k) of row n at position c ^ f(n)
  constexpr int ACH = AROW / 16, WCH = WROW / 16;
  auto fw = [](int n) { return WCH == 16 ? n : (n >> 1) & 7; };
  auto side_group = [](int i, int ln) { const int q = (i * 64 + ln) >> 4; return q < NG ? q : NG - 1; };   // a lane's group of the piece (lanes to spare: the last one)
  // per-lane byte offsets of the loads of a slot of W, of its scales and zero points, where all of them are there
  uint32_t vw[NL], vs[NSL];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int row = i * WRI + lane / WCH;
    vw[i] = (uint32_t)row * (uint32_t)a.ldw + (uint32_t)((lane % WCH) ^ fw(row)) * 16u;
  }
#pragma unroll
  for (int i = 0; i < NSL; ++i) vs[i] = (uint32_t)side_group(i, lane) * (uint32_t)a.lds + (uint32_t)(lane & 15);   // (in numbers)
  // this lane's places in a slot of A (its chunk 4 s + g by XOR, slots begin on 256 bytes) and of W (its word of chunk s)
  const uint32_t a_lane = (uint32_t)((r16 & 3) * AROW + ((g ^ r16) << 4)), w_lane = (uint32_t)(r16 * WROW + (fw(r16) << 4) + 4 * g);
  // without zero points the scales are read in their place, and multiplied by 0
  const uint32_t z_at = a.Z ? SIDE : 0;
  const float z_mul = a.Z ? -1.f : 0.f, z_add = a.Z ? -16.f : -24.f;
  static_assert(W4_RING % 256 == 0 && SIDE % 256 == 0 && BODY % 256 == 0, "...");

  for (int base = 0; base < nblk; base += GB) {
    const int nb = nblk - base < GB ? nblk - base : GB;
    const int S = SA + nb, T = mine * S;
    f32x4 acc[GB][MT];
#pragma unroll
    for (int b = 0; b < GB; ++b)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) acc[b][mt] = f32x4{0.f, 0.f, 0.f, 0.f};

    // the cursor: the next slot of the stream to fetch, f_s of piece f_p, and its place
    int f_t = 0, f_s = 0, f_p = first, issued = 0, need = 0;
    uint32_t f_slot = ring;
    auto fetch = [&]() __attribute__((always_inline)) {
      if (f_t >= T) return;
      const int k0 = f_p * KP;
      const bool tail = k0 + KP > K;                       // chunks past K: the row's first one; they count as zeros
      if (f_s < SA) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          const int row = f_s * 4 + i * ARI;               // (uniform; with two rows a load the second may be one too many: the first again)
          if (row < M) {
            const int in = ARI == 1 ? 0 : lane / ACH;
            int c = (lane % ACH) ^ ((row & 15) + in);
            if (tail && k0 + c * 8 >= K) c = 0;
            load_lds16(A + (int64_t)row * a.lda + k0, (ARI > 1 && in && row + 1 < M ? (uint32_t)a.lda * 2u : 0u) + (uint32_t)c * 16u, f_slot + i * 1024u);
            ++issued;
          }
        }
      } else {
        const int n0 = c0 + (base + f_s - SA) * 16, rows = c1 - n0, g0 = k0 / G;
        const uint8_t* src = a.W + (int64_t)n0 * a.ldw + k0 / 2;
        const uint16_t* sp = a.S + g0 * a.lds + n0;
        const uint8_t* zp = a.Z + g0 * a.ldz + n0;
        if (!tail && rows >= 16) {
#pragma unroll
          for (int i = 0; i < NL; ++i) load_lds16_stream(src, vw[i], f_slot + i * 1024u);
#pragma unroll
          for (int i = 0; i < NSL; ++i) {
            load_lds_u16(sp, vs[i] * 2u, f_slot + BODY + i * 256u);
            if (a.Z) load_lds_u8(zp, vs[i] + (uint32_t)side_group(i, lane) * (uint32_t)(a.ldz - a.lds), f_slot + BODY + SIDE + i * 256u);
          }
        } else {                                           // columns that are not there: the first one's weights, the last one's scales; groups: the last one's
          int ln = lane;
          asm volatile("" : "+v"(ln));
#pragma unroll
          for (int i = 0; i < NL; ++i) {
            const int row = i * WRI + ln / WCH, c = (ln % WCH) ^ fw(row);
            load_lds16_stream(src, row < rows && k0 + c * 32 < K ? (uint32_t)row * (uint32_t)a.ldw + (uint32_t)c * 16u : 0u, f_slot + i * 1024u);
          }
#pragma unroll
          for (int i = 0; i < NSL; ++i) {
            const int n = (ln & 15) < rows ? ln & 15 : rows - 1, qq = side_group(i, ln), q = qq < last_group - g0 ? qq : last_group - g0;
            load_lds_u16(sp, ((uint32_t)q * (uint32_t)a.lds + n) * 2u, f_slot + BODY + i * 256u);
            if (a.Z) load_lds_u8(zp, (uint32_t)q * (uint32_t)a.ldz + n, f_slot + BODY + SIDE + i * 256u);
          }
        }
        issued += a.Z ? NL + 2 * NSL : NL + NSL;
      }
      ++f_t;
      f_slot += slot_bytes;
      if (f_slot == ring_end) f_slot = ring;
      if (++f_s == S) {
        f_s = 0;
        f_p += W4_NW;
      }
    };
#pragma clang loop unroll(disable)
    for (int i = 0; i < slots; ++i) fetch();

    // waits until the next `take` slots, of so many loads, have landed (what was issued after them may be in flight), and gives their places to the next ones
    uint32_t slot = ring;
    auto wait = [&](int loads) __attribute__((always_inline)) {
      need += loads;
      int later = issued - need;
#ifdef MLT_DEBUG_BARRIERS
      later = 0;                                           // waits for all of them, so that a count that is too lax shows
#endif
      if (later >= 16) __builtin_amdgcn_s_waitcnt(wait_imm(16, 15));
      else if (later >= 12) __builtin_amdgcn_s_waitcnt(wait_imm(12, 15));
      else if (later >= 9) __builtin_amdgcn_s_waitcnt(wait_imm(9, 15));
      else if (later >= 6) __builtin_amdgcn_s_waitcnt(wait_imm(6, 15));
      else if (later >= 4) __builtin_amdgcn_s_waitcnt(wait_imm(4, 15));
      else if (later >= 2) __builtin_amdgcn_s_waitcnt(wait_imm(2, 15));
      else __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));
      __builtin_amdgcn_sched_barrier(0);
    };
    auto refill = [&](int take) __attribute__((always_inline)) {
      __builtin_amdgcn_s_waitcnt(wait_imm(63, 0));         // (what was read has arrived)
      __builtin_amdgcn_sched_barrier(0);
#pragma clang loop unroll(disable)
      for (int x = 0; x < take; ++x) {
        fetch();
        __builtin_amdgcn_sched_barrier(0);
        slot += slot_bytes;
        if (slot == ring_end) slot = ring;
      }
    };
    for (int i = 0, piece = first; i < mine; ++i, piece += W4_NW) {
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
          if (WHOLE) {                                     // the ring has room for the tile: each lane reads from its row's slot
            const int take = (rows + 3) / 4;
            wait((rows + ARI - 1) / ARI);
            const uint32_t at = slot + (uint32_t)(r16 < rows ? r16 >> 2 : 0) * (uint32_t)slot_bytes, from = (at >= ring_end ? at - (uint32_t)(slots * slot_bytes) : at) + a_lane;
#pragma unroll
            for (int s = 0; s < NS; ++s) af[mt][s] = *(const MLT_LDS u32x4*)(uintptr_t)((from ^ (uint32_t)((s & 3) << 6)) + (uint32_t)((s >> 2) * 256));
            refill(take);
          } else {                                         // slot by slot
            for (int q = 0; q * 4 < rows; ++q) {
              wait(rows - q * 4 < 4 ? rows - q * 4 : 4);
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
          sa[mt][q] = sum[0];
          asm volatile("" : "+v"(sa[mt][q]));              // (a register of its own: the other three of the four are not to be kept with it)
          __builtin_amdgcn_sched_barrier(0);
        }
      }
#pragma clang loop unroll(disable)
      for (int blk = 0; blk < nb; ++blk) {
        wait(a.Z ? NL + 2 * NSL : NL + NSL);
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
          zp[q & 1] = *(const MLT_LDS u32x4*)(uintptr_t)(slot + BODY + z_at + q * 64u + g * 16u);
        };
        read(0);
#pragma unroll
        for (int q = 0; q < NG; ++q) {
          if (q + 1 < NG) read(q + 1);
          f32x4 sum[MT];
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) sum[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < SPG; ++s) {
            const uint32_t x = w[q & 1][s];
            const u32x4 wf = {nibbles<Tag>(x, 0), nibbles<Tag>(x, 1), nibbles<Tag>(x, 2), nibbles<Tag>(x, 3)};
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) sum[mt] = mfma16(__builtin_bit_cast(V8, wf), __builtin_bit_cast(V8, af[mt][q * SPG + s]), sum[mt]);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float scale = Elem<Tag>::to_f32((uint16_t)sc[q & 1][r]), off = __builtin_fmaf((float)zp[q & 1][r], z_mul, z_add);   // -(16 + z)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) res[mt][r] = __builtin_fmaf(__builtin_fmaf(off, sa[mt][q], sum[mt][r]), scale, res[mt][r]);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int b = 0; b < GB; ++b)
          if (b == blk) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) add4(acc[b][mt], res[mt]);
          }
        refill(1);
      }
    }
    // ---- the wavefronts' sums into their own rings (all their loads have landed), then the sums of those. acc register r: column 4 g + r, row r16 of the tile
    float* own = reinterpret_cast<float*>(smem + wave * W4_RING);
    static_assert(GB * MT * 1024 <= W4_RING, "a wavefront's sums lie in its own ring");
#pragma unroll
    for (int b = 0; b < GB; ++b)
      if (b < nb) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) *reinterpret_cast<f32x4_mem*>(own + (b * MT + mt) * 256 + r16 * 16 + 4 * g) = acc[b][mt];
      }
    __syncthreads();
    for (int e = tid; e < nb * MT * 256; e += W4_NT) {
      const int t = e >> 8, gr = t % MT * 16 + ((e >> 4) & 15), gc = c0 + (base + t / MT) * 16 + (e & 15);
      if (gr < M && gc < c1) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < W4_NW; ++w) sum += reinterpret_cast<const float*>(smem)[w * (W4_RING / 4) + e];
        if (split) store_shared(a.part + ((int64_t)part_id * a.M + m0 + gr) * N + gc, sum);
        else a.C[(int64_t)(m0 + gr) * a.ldc + gc] = Elem<Tag>::from_f32(sum);
      }
    }
    if (base + GB < nblk) __syncthreads();
  }
  if (!split) return;

  // the last part of these columns to get here adds them all (4 elements of a thread at a time, all their parts requested before the first is used)
  if (!last_to_arrive(a.counter + bid * (int)gridDim.z + (int)blockIdx.z, gridDim.y, reinterpret_cast<uint32_t*>(smem))) return;
  const int cols = c1 - c0, parts = (int)gridDim.y;
  const int64_t part_size = (int64_t)a.M * N;
  constexpr int EB = 4;
  for (int e0 = tid; e0 < M * cols; e0 += EB * W4_NT) {
    float v[8][EB];
    int64_t at[EB];
#pragma unroll
    for (int i = 0; i < EB; ++i) {
      const int e = e0 + i * W4_NT < M * cols ? e0 + i * W4_NT : e0;
      at[i] = (int64_t)(m0 + e / cols) * N + c0 + e % cols;
    }
#pragma unroll
    for (int p = 0; p < 8; ++p)
      if (p < parts) {
#pragma unroll
        for (int i = 0; i < EB; ++i) v[p][i] = load_shared(a.part + p * part_size + at[i]);
      }
#pragma unroll
    for (int p = 1; p < 8; ++p)
      if (p < parts) {
#pragma unroll
        for (int i = 0; i < EB; ++i) v[0][i] += v[p][i];
      }
#pragma unroll
    for (int i = 0; i < EB; ++i)
      if (e0 + i * W4_NT < M * cols) {
        const int e = e0 + i * W4_NT;
        a.C[(int64_t)(m0 + e / cols) * a.ldc + c0 + e % cols] = Elem<Tag>::from_f32(v[0][i]);
      }
  }
}

template <typename Tag, int MT, int G, int KP, int GB>
int launch_w4(const W4& a, unsigned nwg, int parts, hipStream_t s) {
  auto kern = gemm_4bit_kernel<Tag, MT, G, KP, GB>;
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
  hipLaunchKernelGGL(kern, dim3(nwg, (unsigned)parts, (unsigned)((a.M + W4_ROWS - 1) / W4_ROWS)), dim3(W4_NT), W4_NW * W4_RING, s, a);
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

template <typename Tag, int G>
int run_w4_rows(const W4& a, unsigned nwg, int parts, hipStream_t s) {
  const int rows = a.M < W4_ROWS ? a.M : W4_ROWS;
  if (rows <= 16) return launch_w4<Tag, 1, G, G == 32 ? 256 : 512, 8>(a, nwg, parts, s);   // (there are no registers for 16 groups)
  if (rows <= 32) return launch_w4<Tag, 2, G, 256, 8>(a, nwg, parts, s);
  return launch_w4<Tag, 4, G, 256, 4>(a, nwg, parts, s);
}

template <typename Tag>
int run_w4_t(const W4& a, int group, unsigned nwg, int parts, hipStream_t s) {
  return group == 32 ? run_w4_rows<Tag, 32>(a, nwg, parts, s) : group == 64 ? run_w4_rows<Tag, 64>(a, nwg, parts, s) : run_w4_rows<Tag, 128>(a, nwg, parts, s);
}

__global__ __launch_bounds__(256) void zero_rows_kernel(uint16_t* C, int64_t ldc, int N) {
  for (int n = (int)blockIdx.x * 256 + threadIdx.x; n < N; n += (int)gridDim.x * 256) C[(int64_t)blockIdx.y * ldc + n] = 0;
}

}  // namespace

int run_gemm_4bit(const Gemm4bitArgs& g, hipStream_t s, char* name, size_t size) {
  if (g.K == 0) {
    snprintf(name, size, "gemm_4bit_zero");
    for (int64_t r = 0; r < g.M; r += 65535) {
      const int64_t n = g.M - r < 65535 ? g.M - r : 65535;
      hipLaunchKernelGGL(zero_rows_kernel, dim3((unsigned)((g.N + 2047) / 2048), (unsigned)n), dim3(256), 0, s, g.C + r * g.ldc, g.ldc, (int)g.N);
      if (hipGetLastError() != hipSuccess) return MLT_ERR_LAUNCH;
    }
    return MLT_OK;
  }
  DeviceInfo di;
  const int64_t ncu = device_info(di) && di.ncu > 0 ? di.ncu : 256;
  const int64_t nz = (g.M + W4_ROWS - 1) / W4_ROWS, rows = g.M < W4_ROWS ? g.M : W4_ROWS;
  // parts of K until a workgroup reads no more of A than of W (2 rows K / parts against columns K / 2 / parts), as long as each wavefront keeps a piece
  int parts = 1;
  const int64_t kp = rows <= 16 && g.group > 32 ? 512 : 256, pieces = (g.K + kp - 1) / kp;
  while (parts < 8 && rows * 4 * ncu > g.N * parts * 2 && pieces >= 2 * parts * W4_NW) parts *= 2;
  while (parts > 1 && (parts * g.M * g.N * 4 > (int64_t)32 << 20 || ncu / parts * nz > kScratchCounters)) parts /= 2;
  float* part = nullptr;
  if (parts > 1) {
    part = cached_scratch(parts * g.M * g.N * 4, s);
    if (!part) parts = 1;
  }
  int64_t nwg = ncu / parts;
  if (nwg > (g.N + 3) / 4) nwg = (g.N + 3) / 4;
  if (nz > 65535 || !launch_fits(nwg * parts * nz, W4_NT)) return MLT_ERR_UNSUPPORTED;
  W4 a{(int)g.M, (int)g.N, (int)g.K, (int)(g.N / nwg), (int)(g.N % nwg), (int)g.lda, (int)g.ldw, g.A, g.W, g.S, g.Z, g.lds, g.ldz, g.C, g.ldc, part,
       part ? scratch_counters(part) : nullptr};
  snprintf(name, size, "gemm_4bit_g%d_m%d_parts%d", (int)g.group, rows <= 16 ? 16 : rows <= 32 ? 32 : 64, parts);
  return g.dtype == MLT_BF16 ? run_w4_t<bf16_tag>(a, (int)g.group, (unsigned)nwg, parts, s) : run_w4_t<f16_tag>(a, (int)g.group, (unsigned)nwg, parts, s);
}

}  // namespace mlt
