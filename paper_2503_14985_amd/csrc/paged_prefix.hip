// Single-token attention of a batch whose sequences share a prefix (mlt_paged_attn_decode_prefix): one query per (sequence, query head), G = Hq / H query heads to a key/value head.
//
// The prefix is read once for all sequences: the B G queries of a key/value head are the rows of one matrix, against the prefix's keys. Each sequence's own keys follow, for its G
// queries alone. Both leave a maximum, a sum and an output that is not divided yet (fp32), which a second kernel joins in a fixed order. One launch does both kinds of
// work: the prefix is bound by the matrix units, the own keys by memory, and CUs that are busy with the one leave the other what it is short of.
//   * The prefix of more than 32 rows: tiles of 256 rows and 64 keys (prompt_body in prompt_tile.h), its keys cut into ranges.
//   * Own keys, and the prefix of up to 32 rows: nothing is shared, so reading the cache (4 D bytes a key and head) is the cost. A wavefront has an LDS ring of its own with room for the rows of one
//     unit of 32 keys, which it fills by direct loads of 1 KB of whole rows and waits for by count (K of the next unit is asked for as soon as this one's K is in
//     registers, then V); no barrier until the end. S^T = K Q^T and O^T = V^T P^T on 16x16x32 MFMAs with the queries as the 16 columns. S^T leaves key 4 (l / 16) + r of
//     query l % 16 in register r, which are k slots 8 (l / 16) .. + 7 of the second product (four from each half of 16 keys): P needs no exchange between lanes, and the
//     transposing LDS read fetches V for the same keys. P goes in as the sum of two 16-bit numbers, itself rounded and what that left (16 bits of bf16, 22 of fp16): the matrix
//     units have time for it. Its sum is taken in fp32 before the rounding.
// 64 sequences, 32 heads over 8, D = 128, behind a prefix of 8192 with up to 512 own keys: 35 us (29 here, of which a third is the partial results of 17 ranges; 6 in joining them); 250 behind 32001: 150 to 157 us, the
// rate of the prompts' kernel; 64 behind 1024 with up to 4096 own keys: 120 us, 5.6 TB/s. Ranges of 8 key tiles at least: with 4 the first takes 53 us, with 12 35, but 16 sequences behind 4096 keys 25 instead of 21.
// Short prefixes are not shared at all (plan_prefix). A sequence that ends inside the prefix is not part of it: all of its keys, up to its end, are its own, read through the prefix's table. So are they where there is no room for
// partial results.
#include <stdio.h>

#include "fp8.h"
#include "prompt_tile.h"

namespace mlt {

namespace {

constexpr int PX_UNIT = 32, PX_NW = 8, PX_NT = PX_NW * 64;
constexpr int PX_MAX_PARTS = 64;           // partial results of a query, at most
constexpr float PX_LAZY = 8.f, PX_GAIN = 6.f;   // log2: what a maximum may grow before the reference moves; what weights are multiplied by (fp16's small end)

template <int D> struct PxRing {
  static constexpr int ROWB = 2 * D, CPR = D / 8, RPB = 64 / CPR;         // bytes and 16-byte chunks of a row, rows of a load
  static constexpr int MAT = PX_UNIT * ROWB, NLD = MAT / 1024;            // bytes of a unit's keys (or values), loads of them
  static constexpr int WAVE = 2 * MAT + 256;                              // a unit, and block numbers for 32 units
  static constexpr int SMEM = PX_NW * WAVE;
  // chunk c of row r lies at position c ^ f(r): rows read together (16 of K at one chunk; 8 of V at two) in different banks
  static __device__ __forceinline__ int fk(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
  static __device__ __forceinline__ int fv(int r) { return D == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3); }
};

struct Prefix {
  const uint16_t *Q, *Kc, *Vc;
  const int32_t *prefix_table, *block_table, *seq_lens;
  uint16_t* O;
  float *part_o, *part_s;      // [query][parts][D], [query][parts][2]; null: one part, straight to O
  int B, H, G, block_size, max_blocks, num_blocks, P;
  int nxcd, tiles;             // tiles of 16 queries of a group
  int pre_parts, own_parts;    // ranges of the prefix (0: every sequence reads it), of the own keys
  int pre_tiles, pre_per;      // row tiles of the prefix; key tiles (units) of a range
  int pre_blocks;              // workgroups for it
  int waves;                   // wavefronts of an item of own keys
  float c;
};

// Queries of rows r0 .. r0 + nq - 1 (row: sequence * G + head of the group) of key/value head h, over one or two runs of keys: na halves of 16 keys of the prefix's table, keys 0 .. a_end - 1
// of them, then nb halves from half b0 of `table`, keys b_begin .. b_end - 1. Units u0 + wave, + waves, ... of 32 keys up to u1.
struct PxItem {
  int h, r0, nq;
  int na, a_end, nb, b0, b_begin, b_end;
  const int32_t* table;
  int u0, u1;
};

template <typename Tag, int D, int NQT>
__device__ __forceinline__ void px_ring(const Prefix& a, const PxItem& it, int wave_in, int waves, uint32_t ring, float (&m)[NQT], float (&l)[NQT], f32x4 (&o)[NQT][D / 16]) {
  typedef PxRing<D> L;
  typedef typename Elem<Tag>::vec8 V8;
  constexpr int NT = D / 16, KP = D / 32, NLD = L::NLD, ROWB = L::ROWB;
  const int lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4;
  const int halves = it.na + it.nb, hpb = a.block_size / 16;
  const int mine = it.u1 > it.u0 + wave_in ? (it.u1 - it.u0 - wave_in + waves - 1) / waves : 0;

  // Q^T fragments: dimensions 32 i + 8 g .. + 7 of query r16 of each tile
  V8 qf[NQT][KP];
#pragma unroll
  for (int q = 0; q < NQT; ++q) {
    const int r = 16 * q + r16 < it.nq ? it.r0 + 16 * q + r16 : it.r0, b = r / a.G;
    const uint16_t* qp = a.Q + ((int64_t)b * (a.H * a.G) + it.h * a.G + (r - b * a.G)) * D + 8 * g;
#pragma unroll
    for (int i = 0; i < KP; ++i) qf[q][i] = __builtin_bit_cast(V8, *reinterpret_cast<const u32x4_mem*>(qp + 32 * i));
  }
#pragma unroll
  for (int q = 0; q < NQT; ++q) {
    m[q] = -__builtin_inff();
    l[q] = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t) o[q][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  if (mine == 0) return;

  // Where the halves lie: lane 2 i + p holds that of half p of the wavefront's i-th unit, 32 units at a time (halves past the last one: that again), in 16 rows. The next 32 are
  // looked up, through LDS and in the stream of the other loads, while these are worked on.
  auto entry = [&](int first) __attribute__((always_inline)) {             // this lane's half, of units first, first + waves, ...
    const int v = 2 * (first + lane / 2 * waves) + (lane & 1);
    return v < halves ? v : halves - 1;
  };
  auto table_at = [&](int v) __attribute__((always_inline)) { return v < it.na ? a.prefix_table + v / hpb : it.table + (it.b0 + v - it.na) / hpb; };
  auto place = [&](int v, int blk) __attribute__((always_inline)) {        // (the host checks that it fits)
    blk = blk < 0 ? 0 : blk >= a.num_blocks ? a.num_blocks - 1 : blk;
    return (uint32_t)((blk * a.H + it.h) * hpb + (v < it.na ? v : it.b0 + v - it.na) % hpb);
  };
  const uint32_t side = ring + 2 * L::MAT;
  constexpr int NK = D == 128 ? 4 : 2, NV = D == 128 ? 2 : 1;              // loads differ in their rows' swizzles
  uint32_t vk[NK], vv[NV];
  const int in = lane / L::CPR, slot = lane % L::CPR;
#pragma unroll
  for (int j = 0; j < NK; ++j) vk[j] = (uint32_t)(in * ROWB + (slot ^ L::fk(L::RPB * j + in)) * 16);
#pragma unroll
  for (int j = 0; j < NV; ++j) vv[j] = (uint32_t)(in * ROWB + (slot ^ L::fv(L::RPB * j + in)) * 16);
  auto fetch = [&](const uint16_t* mat, bool v, uint32_t at, int i, uint32_t dst) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NLD; ++j) {
      const int p = j * 2 / NLD, part = j % (NLD / 2);                     // half, and 1 KB of it
      const char* row0 = reinterpret_cast<const char*>(mat) + (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)at, 2 * i + p) * (16 * ROWB) + part * 1024;
      load_lds16_stream(row0, v ? vv[part % NV] : vk[part % NK], dst + j * 1024);
    }
  };
  const uint32_t k_at = (uint32_t)(r16 * ROWB + ((g ^ L::fk(r16)) << 4));
  const int vrow = 4 * g + (r16 >> 2);
  const uint32_t v_at = (uint32_t)(L::MAT + vrow * ROWB + ((((r16 & 3) >> 1) ^ L::fv(vrow)) << 4) + 8 * (r16 & 1));

  auto landed = [&](auto n) __attribute__((always_inline)) {
#ifdef MLT_DEBUG_BARRIERS
    __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));
#else
    __builtin_amdgcn_s_waitcnt(wait_imm(decltype(n)::value, 15));
#endif
    __builtin_amdgcn_sched_barrier(0);
  };
  auto lds_read = [&]() __attribute__((always_inline)) {  // the reads so far are done: what they read may be overwritten
    __builtin_amdgcn_s_waitcnt(wait_imm(63, 0));
    __builtin_amdgcn_sched_barrier(0);
  };

  uint32_t at, next_at = 0;
  {
    const int v = entry(it.u0 + wave_in);
    at = place(v, *table_at(v));
    // (here, so that the compiler waits for the queries before the loop and not, with all that is in flight, in it)
#pragma unroll
    for (int q = 0; q < NQT; ++q)
#pragma unroll
      for (int i = 0; i < KP; ++i) asm volatile("" : "+v"(qf[q][i]));
    fetch(a.Kc, false, at, 0, ring);
    fetch(a.Vc, true, at, 0, ring + L::MAT);
  }
#pragma clang loop unroll(disable)
  for (int i = 0; i < mine; ++i) {
    const int j = i & 31, u = it.u0 + wave_in + i * waves;
    const bool more = i - j + 32 < mine;                 // units behind these 32
    if (j == 4 && more) load_lds4(table_at(entry(u + 28 * waves)), side);
    // ---- scores. Since the loads of K: those of V
    landed(std::integral_constant<int, NLD>{});
    if (j == 16 && more) {                               // (the block numbers were asked for twelve units ago)
      const int v = entry(u + 16 * waves);
      next_at = place(v, *(const MLT_LDS int*)(uintptr_t)(side + lane * 4u));
      lds_read();
    }
    u32x4 kr[2][KP];
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int c = 0; c < KP; ++c) kr[p][c] = *(const MLT_LDS u32x4*)(uintptr_t)(ring + (uint32_t)(p * 16 * ROWB) + (k_at ^ (uint32_t)(c * 64)));
    lds_read();
    if (j == 31) at = next_at;                           // from here on units i + 1 and later are fetched
    if (i + 1 < mine) fetch(a.Kc, false, at, (i + 1) & 31, ring);
    // the halves' first keys and what counts of them
    int first[2], lo[2], hi[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int v = 2 * u + p;
      first[p] = 16 * (v < it.na ? v : it.b0 + v - it.na);
      lo[p] = v < it.na ? 0 : it.b_begin;
      hi[p] = v < it.na ? it.a_end : v < halves ? it.b_end : 0;
    }
    const bool cut = first[0] < lo[0] || first[1] < lo[1] || first[0] + 16 > hi[0] || first[1] + 16 > hi[1];
    u32x4 pf[NQT], pl[NQT];                              // P rounded, and what that left
#pragma unroll
    for (int q = 0; q < NQT; ++q) {
      float s[2][4];
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KP; ++c) acc = mfma16(__builtin_bit_cast(V8, kr[p][c]), qf[q][c], acc);
#pragma unroll
        for (int r = 0; r < 4; ++r) s[p][r] = acc[r] * a.c;
      }
      if (cut) {                                         // keys that do not count: no weight, whatever lies there
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int key = first[p] + 4 * g + r;
            if (key < lo[p] || key >= hi[p]) s[p][r] = -__builtin_inff();
          }
      }
      float mx = __builtin_fmaxf(max3(s[0][0], s[0][1], s[0][2]), max3(s[0][3], s[1][0], s[1][1]));
      mx = max3(mx, s[1][2], s[1][3]);
      if (__any(mx > m[q] + PX_LAZY)) {                  // (m = -inf: the first time)
        mx = __builtin_fmaxf(mx, __shfl_xor(mx, 16));
        mx = __builtin_fmaxf(mx, __shfl_xor(mx, 32));
        const float now = __builtin_fmaxf(m[q], mx);
        if (now > -__builtin_inff()) {                   // (else nothing has been added yet)
          const float alpha = __builtin_amdgcn_exp2f(m[q] - now);
          l[q] *= alpha;
          m[q] = now;
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[q][t][r] *= alpha;
        }
      }
      const float ref = m[q] == -__builtin_inff() ? 0.f : m[q];
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        float e[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          e[r] = __builtin_amdgcn_exp2f(s[p][r] - ref + PX_GAIN);
          l[q] += e[r];
        }
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
          const uint32_t w = Elem<Tag>::pack2(e[r], e[r + 1]);
          pf[q][2 * p + r / 2] = w;
          pl[q][2 * p + r / 2] = Elem<Tag>::pack2(e[r] - Elem<Tag>::to_f32((uint16_t)w), e[r + 1] - Elem<Tag>::to_f32((uint16_t)(w >> 16)));
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    // ---- outputs. Since the loads of V: those of K of the next unit
    if (i + 1 < mine) landed(std::integral_constant<int, NLD>{}); else landed(std::integral_constant<int, 0>{});
    u32x4 vr[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const uint32_t at_t = ring + (v_at ^ (uint32_t)(t * 32));
      const s16x4 h0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((MLT_LDS s16x4*)(uintptr_t)at_t);
      const s16x4 h1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((MLT_LDS s16x4*)(uintptr_t)(at_t + 16 * ROWB));
      vr[t] = __builtin_bit_cast(u32x4, __builtin_shufflevector(h0, h1, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    lds_read();
    if (i + 1 < mine) fetch(a.Vc, true, at, (i + 1) & 31, ring + L::MAT);
    if (cut) {
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
          const int key = first[p] + 4 * g + r;
          const uint32_t keep = (key >= lo[p] && key < hi[p] ? 0xffffu : 0u) | (key + 1 >= lo[p] && key + 1 < hi[p] ? 0xffff0000u : 0u);
#pragma unroll
          for (int t = 0; t < NT; ++t) vr[t][2 * p + r / 2] &= keep;
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int q = 0; q < NQT; ++q) {
        o[q][t] = mfma16(__builtin_bit_cast(V8, vr[t]), __builtin_bit_cast(V8, pf[q]), o[q][t]);
        o[q][t] = mfma16(__builtin_bit_cast(V8, vr[t]), __builtin_bit_cast(V8, pl[q]), o[q][t]);
      }
  }
#pragma unroll
  for (int q = 0; q < NQT; ++q) {
    l[q] += __shfl_xor(l[q], 16);
    l[q] += __shfl_xor(l[q], 32);
    m[q] -= PX_GAIN;                                     // what l and o are relative to
  }
}

// The results of the `waves` wavefronts of each item of a workgroup meet in LDS, a tile of 16 queries at a time, and leave: as part number `part` of its query's results, or divided. items: of this workgroup.
template <typename Tag, int D, int NQT>
__device__ __forceinline__ void px_store(const Prefix& a, const PxItem& it, char* smem, int waves, int part, bool there, const float (&m)[NQT], const float (&l)[NQT],
                                         const f32x4 (&o)[NQT][D / 16]) {
  constexpr int LD = D + 4, NT = D / 16;
  const int lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4, wave = uniform((int)threadIdx.x >> 6);
  float *sm = reinterpret_cast<float*>(smem), *sl = sm + PX_NW * 16, *so = sl + PX_NW * 16;
  const int w0 = wave / waves * waves, sub = (int)threadIdx.x - w0 * 64, threads = waves * 64;
#pragma unroll
  for (int q = 0; q < NQT; ++q) {
    __syncthreads();                                     // (everybody is past its ring, or the tile before)
    if (g == 0) {
      sm[wave * 16 + r16] = m[q];
      sl[wave * 16 + r16] = l[q];
    }
    // register r of tile t is dimension 16 t + 4 g + r
#pragma unroll
    for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4_mem*>(so + (wave * 16 + r16) * LD + 16 * t + 4 * g) = o[q][t];
    __syncthreads();
    const int n = there ? (it.nq - 16 * q < 16 ? it.nq - 16 * q : 16) : 0;
    for (int e = sub; e < n * (D / 4); e += threads) {
      const int r = e / (D / 4), d = e % (D / 4) * 4;
      float M = -__builtin_inff(), S = 0.f;
      for (int w = 0; w < waves; ++w) M = __builtin_fmaxf(M, sm[(w0 + w) * 16 + r]);
      const float ref = M == -__builtin_inff() ? 0.f : M;    // no key at all: sums and outputs are zeros
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
      for (int w = 0; w < waves; ++w) {
        const float wgt = __builtin_amdgcn_exp2f(sm[(w0 + w) * 16 + r] - ref);
        S += sl[(w0 + w) * 16 + r] * wgt;
        const f32x4 x = *reinterpret_cast<const f32x4_mem*>(so + ((w0 + w) * 16 + r) * LD + d);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] += x[i] * wgt;
      }
      const int row = it.r0 + 16 * q + r, b = row / a.G;
      const int64_t query = (int64_t)b * (a.H * a.G) + it.h * a.G + (row - b * a.G);
      if (a.part_o) {
        const int64_t at = query * (a.pre_parts + a.own_parts) + part;
        if (d == 0) { a.part_s[2 * at] = M; a.part_s[2 * at + 1] = S; }
        *reinterpret_cast<f32x4_mem*>(a.part_o + at * D + d) = acc;
      } else {
        const float inv = S == 0.f ? 0.f : 1.f / S;
        uint16_t* out = a.O + query * D + d;
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = Elem<Tag>::from_f32(acc[i] * inv);
      }
    }
  }
}

// PRE: 0 no prefix of its own; 1, 2: its rows are one or two tiles of 16; 3: tiles of 256
template <typename Tag, int D, int PRE>
__global__ __launch_bounds__(PX_NT, 2) void paged_prefix_kernel(Prefix a) {
  extern __shared__ __align__(16) char smem[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lptr_t)smem;
  const int wave = uniform((int)threadIdx.x >> 6);
  int id = (int)blockIdx.x;
  if (PRE == 3 && id < a.pre_blocks) {
    // row tiles of one head and range side by side on an XCD, which reads that range's keys from memory once
    id = logical_block(id, a.pre_blocks, a.nxcd);
    const int tile = id % a.pre_tiles, hr = id / a.pre_tiles, range = hr % a.pre_parts, h = hr / a.pre_parts;
    PromptSeq seq{0, a.B, 0, a.P};
    PromptKernel p{a.Q, nullptr, PromptKeys{a.Kc, a.Vc, 0, 0, a.prefix_table, a.block_size, 0, a.num_blocks}, PromptItems{}, (int64_t)a.H * a.G * D, 0, a.c < 0 ? -a.c : a.c, a.c < 0 ? 1 : 0};
    p.c = p.c < 1e-30f ? 1e-30f : p.c;                   // (as in launch_mha_pp)
    p.items.H = a.H;
    p.items.G = a.G;
    prompt_body<Tag, D, false, true, true>(p, seq, 0, h, tile, lds0, PromptPart{range * a.pre_per, a.pre_per, range, a.pre_parts + a.own_parts, a.part_o, a.part_s});
    return;
  }
  const uint32_t ring = lds0 + (uint32_t)wave * PxRing<D>::WAVE;
  if ((PRE == 1 || PRE == 2) && id < a.pre_blocks) {
    constexpr int NQT = PRE == 2 ? 2 : 1;
    const int range = id % a.pre_parts, h = id / a.pre_parts, units = (a.P + PX_UNIT - 1) / PX_UNIT, u0 = range * a.pre_per, u1 = u0 + a.pre_per < units ? u0 + a.pre_per : units;
    const PxItem it{h, 0, a.B * a.G, (a.P + 15) / 16, a.P, 0, 0, 0, 0, nullptr, u0, u1};
    float m[NQT], l[NQT];
    f32x4 o[NQT][D / 16];
    px_ring<Tag, D, NQT>(a, it, wave, PX_NW, ring, m, l, o);
    px_store<Tag, D, NQT>(a, it, smem, PX_NW, range, true, m, l, o);
    return;
  }
  // own keys: an item for each (sequence, key/value head, tile of 16 queries, range), `waves` wavefronts each
  const int items_per = PX_NW / a.waves;
  int item = (PRE ? id - a.pre_blocks : id) * items_per + wave / a.waves;
  const int all = a.B * a.H * a.tiles * a.own_parts;
  const bool there = item < all;
  item = there ? item : all - 1;
  const int range = item % a.own_parts;
  item /= a.own_parts;
  const int tile = item % a.tiles, bh = item / a.tiles, b = uniform(bh / a.H), h = bh - b * a.H;
  const int cap = a.max_blocks * a.block_size;
  int len = a.seq_lens[b];
  len = len < 0 ? 0 : len > cap ? cap : len;
  PxItem it;
  it.h = uniform(h);
  it.r0 = b * a.G + 16 * tile;
  it.nq = a.G - 16 * tile < 16 ? a.G - 16 * tile : 16;
  const bool shared = a.pre_parts > 0 && len >= a.P;     // the prefix's part is done for this sequence
  it.a_end = len < a.P ? len : a.P;
  it.na = shared ? 0 : (it.a_end + 15) / 16;
  it.b0 = a.P / 16;
  it.b_begin = a.P;
  it.b_end = len;
  it.nb = len > a.P ? (len + 15) / 16 - it.b0 : 0;
  it.table = a.block_table + (int64_t)b * a.max_blocks;
  const int units = (it.na + it.nb + 1) / 2, per = ((units + a.own_parts - 1) / a.own_parts + a.waves - 1) / a.waves * a.waves;
  it.u0 = range * per;
  it.u1 = it.u0 + per < units ? it.u0 + per : units;
  float m[1], l[1];
  f32x4 o[1][D / 16];
  px_ring<Tag, D, 1>(a, it, wave % a.waves, a.waves, ring, m, l, o);
  px_store<Tag, D, 1>(a, it, smem, a.waves, a.pre_parts + range, there, m, l, o);
}

// The parts of each query, in their order: first the prefix's (unless the sequence ends inside it), then its own. 4 D / 4 threads to a query: D / 4 lanes with 4 elements each, 4 groups of them every fourth part.
template <typename Tag, int D>
__global__ __launch_bounds__(256) void paged_prefix_merge_kernel(const float* __restrict__ part_o, const float* __restrict__ part_s, const int32_t* __restrict__ seq_lens,
                                                                  uint16_t* __restrict__ O, int Hq, int P, int pre_parts, int parts, int64_t queries) {
  constexpr int LQ = D / 4, QPW = 256 / (4 * LQ);        // lanes across the elements, queries of a workgroup
  const int tid = threadIdx.x, d = tid % LQ * 4, grp = tid / LQ % 4;
  const int64_t query = (int64_t)blockIdx.x * QPW + tid / (4 * LQ);
  const bool there = query < queries;
  const int64_t q = there ? query : queries - 1;
  const int first = seq_lens[q / Hq] >= P ? 0 : pre_parts;
  // lane i: maximum and sum of part i (at most 64), none if it is not to be read or had no keys (NaN scores leave a maximum of -inf too, but a sum of NaN)
  const int lane = tid & 63;
  float mi = -__builtin_inff(), si = 0.f;
  if (lane >= first && lane < parts) {
    mi = part_s[(q * parts + lane) * 2];
    si = part_s[(q * parts + lane) * 2 + 1];
  }
  const unsigned long long some = __ballot(!(mi == -__builtin_inff() && si == 0.f));
  const float M = wave_max(mi), ref = M == -__builtin_inff() ? 0.f : M, wi = __builtin_amdgcn_exp2f(mi - ref);
  const float* so = part_o + q * parts * D + d;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float S = 0.f;
  for (int i0 = 0; i0 < parts; i0 += 16) {               // four parts of a group's turn at once; all lanes stay, they hold the parts' weights
    f32x4 x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = i0 + grp + 4 * k;
      x[k] = *reinterpret_cast<const f32x4_mem*>(so + (int64_t)(i < parts ? i : parts - 1) * D);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = i0 + grp + 4 * k;
      const float w = __shfl(wi, i & 63), s = __shfl(si, i & 63);
      if (i < parts && (some >> i & 1)) {
        S += s * w;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += x[k][e] * w;
      }
    }
  }
  __shared__ f32x4 buf[256];
  __shared__ float sums[256];
  buf[tid] = acc;
  sums[tid] = S;
  __syncthreads();
  if (grp != 0 || !there) return;
#pragma unroll
  for (int i = 1; i < 4; ++i) {
    add4(acc, buf[tid + i * LQ]);
    S += sums[tid + i * LQ];
  }
  const float inv = S == 0.f ? 0.f : 1.f / S;
  uint16_t* out = O + q * D + d;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = Elem<Tag>::from_f32(acc[e] * inv);
}

struct PrefixPlan { int pre, pre_parts, pre_per, pre_tiles, own_parts, waves; };

// What a plan takes, in us, as far as one can tell from the largest lengths: `blocks` workgroups in rounds, each of some start and end and of its wavefronts' units one after the other; fitted to 1 to 250
// sequences with 300 to 32000 keys in front and 64 to 8192 of their own.
double px_time(int64_t blocks, int64_t units, int64_t D, int64_t ncu) {
  const int64_t places = D == 64 ? 2 * ncu : ncu;
  return (double)((blocks + places - 1) / places) * (2.5 + (D == 64 ? 0.7 : 1.3) * (double)units);
}

// Wavefronts of an item of own keys, and into how many ranges those are cut, for `left` units of 32 keys beside `others` workgroups; merged: there is a second kernel anyway. 512 items of 17 units beside 128 workgroups
// with 2, 4, 8 wavefronts: 37.4, 39.6, 40.9 us in all; 512 of 129: 171, 128, 123.
double plan_own(PrefixPlan& p, int64_t items, int64_t left, int64_t others, bool merged, int64_t D, int64_t ncu) {
  double best = 0.;
  for (int w = 8; w >= 2; w /= 2)
    for (int n = 1; n <= PX_MAX_PARTS / 2 && (n == 1 || (n * 2 * w <= left && items * n <= 4 * ncu)); n *= 2) {
      const double t = px_time((items * n * w + PX_NW - 1) / PX_NW + others, (left + w * n - 1) / (w * n), D, ncu) + (n > 1 ? 0.1 * n + (merged ? 0. : 3.5) : 0.);
      if (best == 0. || t < best) {
        best = t;
        p.waves = w;
        p.own_parts = n;
      }
    }
  return best;
}

double larger(double x, double y) { return x > y ? x : y; }

PrefixPlan plan_prefix(const PrefixArgs& a, int64_t ncu) {
  PrefixPlan p{0, 0, 0, 0, 1, 8};
  const int64_t G = a.Hq / a.H, rows = a.B * G, tiles = (G + 15) / 16, own = a.max_blocks * a.block_size - a.prefix_len;
  const int64_t items = a.B * a.H * tiles, units = (own + 31) / 32 + 1;
  const int64_t pre_units = (a.prefix_len + 31) / 32;
  const double unit = (double)(items * 128 * a.D) * 1e-6;            // MB of a unit of all items: own keys come at 5 TB/s, the prefix's, read by all, mostly from the L2
  const double alone = larger(plan_own(p, items, units + pre_units, 0, false, a.D, ncu), unit * ((double)units / 5. + (double)pre_units / 12.));
  if (a.prefix_len == 0 || a.B == 1) return p;
  // the prefix once for all
  PrefixPlan q{0, 0, 0, 0, 1, 8};
  q.pre = rows <= 16 ? 1 : rows <= 32 ? 2 : 3;
  const int64_t step = q.pre == 3 ? 64 : 32 * PX_NW, steps = (a.prefix_len + step - 1) / step;     // a key tile; a unit for every wavefront
  q.pre_tiles = q.pre == 3 ? (int)((rows + 255) / 256) : 1;
  int64_t n = ncu / (a.H * q.pre_tiles);
  const int64_t least = q.pre == 3 ? 8 : 1;
  if (n > steps / least) n = steps / least;
  if (n > PX_MAX_PARTS / 2) n = PX_MAX_PARTS / 2;
  if (n < 1) n = 1;
  const int64_t per = (steps + n - 1) / n, blocks = (steps + per - 1) / per * q.pre_tiles * a.H;
  q.pre_parts = (int)((steps + per - 1) / per);
  q.pre_per = (int)(q.pre == 3 ? per : per * PX_NW);
  const double theirs = larger(plan_own(q, items, units, blocks, true, a.D, ncu), unit * (double)units / 5.);
  const double shared = q.pre == 3 ? (4. + (a.D == 64 ? 0.9 : 1.7) * (double)per) * (double)((blocks + ncu - 1) / ncu) : px_time(blocks, per, a.D, ncu);
  // Every sequence reads the prefix by itself, in one launch, where that is not slower: 16 sequences behind 500 keys 7.7 us (16.9 shared), 32 behind 1000 11.3 (18.8), 64 behind 500 13.9 (23.2),
  // but 4 behind 1000 9.8 (9.1), 8 behind 2000 13.5 (12.8), and 128 behind 300 are taken for 22.2 shared, 19.1 alone.
  return alone <= larger(theirs, shared) + (q.pre == 3 ? 5. : 4.2) ? p : q;
}
int64_t work_of(const PrefixArgs& a, const PrefixPlan& p) {
  const int64_t parts = p.pre_parts + p.own_parts;
  return parts > 1 ? a.B * a.Hq * parts * (a.D + 2) * 4 : 0;
}
int64_t cus() {
  DeviceInfo di;
  return device_info(di) && di.ncu > 0 ? di.ncu : 256;
}

template <typename Tag, int D, int PRE>
int launch_prefix(const Prefix& a, int64_t grid, hipStream_t s) {
  auto kern = paged_prefix_kernel<Tag, D, PRE>;
  constexpr int RING = PxRing<D>::SMEM, MERGE = (2 * PX_NW * 16 + PX_NW * 16 * (D + 4)) * 4, TILES = PRE == 3 ? PaCfg<D>::SMEM : 0;
  constexpr int LDS = RING > MERGE ? (RING > TILES ? RING : TILES) : (MERGE > TILES ? MERGE : TILES);
  static thread_local int configured_dev = -1;           // opt in to > 64 KB LDS once per device
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return MLT_ERR_DEVICE;
  if (configured_dev != dev) {
    if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, LDS) != hipSuccess) {
      (void)hipGetLastError();
      return MLT_ERR_LAUNCH;
    }
    configured_dev = dev;
  }
  hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(PX_NT), LDS, s, a);
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

template <typename Tag, int D>
int run_prefix_t(const PrefixArgs& g, PrefixPlan p, float* work, hipStream_t s) {
  Prefix a{g.Q, g.Kc, g.Vc, g.prefix_table, g.block_table, g.seq_lens, g.O, nullptr, nullptr, (int)g.B, (int)g.H, (int)(g.Hq / g.H), (int)g.block_size, (int)g.max_blocks, (int)g.num_blocks,
           (int)g.prefix_len, device_xcds(), (int)((g.Hq / g.H + 15) / 16), p.pre_parts, p.own_parts, p.pre_tiles, p.pre_per, p.pre_parts * p.pre_tiles * (int)g.H, p.waves,
           g.scale * 1.4426950408889634f};
  const int64_t parts = p.pre_parts + p.own_parts, queries = g.B * g.Hq;
  if (work) {
    a.part_o = work;
    a.part_s = work + queries * parts * D;
  }
  const int64_t items = g.B * g.H * a.tiles * p.own_parts, grid = a.pre_blocks + (items * p.waves + PX_NW - 1) / PX_NW;
  if (!launch_fits(grid, PX_NT) || !launch_fits(queries, 256)) return MLT_ERR_UNSUPPORTED;
  int rc;
  switch (p.pre) {
    case 1: rc = launch_prefix<Tag, D, 1>(a, grid, s); break;
    case 2: rc = launch_prefix<Tag, D, 2>(a, grid, s); break;
    case 3: rc = launch_prefix<Tag, D, 3>(a, grid, s); break;
    default: rc = launch_prefix<Tag, D, 0>(a, grid, s);
  }
  if (rc != MLT_OK || !work) return rc;
  constexpr int QPW = 256 / D;
  hipLaunchKernelGGL((paged_prefix_merge_kernel<Tag, D>), dim3((unsigned)((queries + QPW - 1) / QPW)), dim3(256), 0, s, a.part_o, a.part_s, g.seq_lens, g.O, (int)g.Hq, (int)g.prefix_len,
                     p.pre_parts, (int)parts, queries);
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

}  // namespace

int64_t paged_prefix_work(const PrefixArgs& a) { return work_of(a, plan_prefix(a, cus())); }

int run_paged_prefix(const PrefixArgs& a, hipStream_t s, char* name, size_t size) {
  PrefixPlan p = plan_prefix(a, cus());
  const int64_t need = work_of(a, p);
  float* work = nullptr;
  ScratchTurn turn;
  if (need > 0) {
    work = a.work ? (a.work_bytes >= need ? a.work : nullptr) : cached_scratch(need, s, turn);
    if (!work) {                                         // everything to one item for each sequence and head
      p = PrefixPlan{0, 0, 0, 0, 1, 8};
    }
  }
  static const char* const kinds[4] = {"", "_16", "_32", "_256"};
  snprintf(name, size, "paged_prefix_d%d%s_p%d_o%dw%d", (int)a.D, kinds[p.pre], p.pre_parts, p.own_parts, p.waves);
  if (a.dtype == MLT_BF16) return a.D == 128 ? run_prefix_t<bf16_tag, 128>(a, p, work, s) : run_prefix_t<bf16_tag, 64>(a, p, work, s);
  return a.D == 128 ? run_prefix_t<f16_tag, 128>(a, p, work, s) : run_prefix_t<f16_tag, 64>(a, p, work, s);
}

}  // namespace mlt
