// Decode attention over a paged cache in e4m3 with a scale for each (block, head): one query per (sequence, query head), G = Hq / H
// query heads to a key/value head.
//
// Reading the cache is the cost (2 * D bytes a key and head), and the G queries that share it go through it together, up to 16 of
// them as the 16 columns of an MFMA: S^T = K Q^T and O^T = V^T P^T, both with the cache as the first operand.
//   * A unit is two halves of 16 keys. A wavefront has an LDS ring of its own with room for the rows of one unit, which it fills by direct loads of
//     1 KB of whole rows and waits for by count (K of the next unit is asked for as soon as this one's K is in registers, then V); no barrier until
//     the end. Fragments loaded from memory into registers, 16 rows x 64 bytes an instruction for K, came at 4.9 TB/s. Room for 2, 4 or 8 units with
//     fewer wavefronts on a CU was slower at every size: what counts is how many wavefronts are there to issue loads, 16 on a CU.
//     Chunk c of row r lies at position c ^ f(r), f such that the rows read together fall in different banks.
//   * K: lane l reads pieces l / 16 of key l % 16 of a half, turned into the 16-bit type of Q (exact). Which k slot of the MFMA a
//     dimension gets is free as long as Q's fragment agrees.
//   * S^T leaves key 4 (l / 16) + r of query l % 16 in register r. Those are the k slots 8 (l / 16) .. + 7 of the second product
//     (four from each half), so P needs no exchange between lanes, and the transposing LDS read fetches V for the same keys.
// P and V are multiplied as fp16 whatever Q's type: e4m3 is exact in it. The scale of V goes into P: p = 2^(score - m - top) * (scale of V), m + top the running maximum of the
// product's log2 over the wavefront's keys (it moves only when a product passes it by 8), so that a large scale on keys of little weight takes no bits from the
// others. p is at most 2^8, 2^6 on top leaves it far from fp16's small end. It goes in as the sum of two fp16 numbers, itself rounded and what that left: 22 bits, as
// good as fp32 beside the output's rounding, for 1 % of the time (64 sequences of up to 4096 keys 55.8 -> 56.4 us, one of 32768 17.0 -> 17.2; the matrix units are idle
// for nine tenths of it), where one of 11 bits made fp16 results a third worse than an fp32 computation's. The weights' sum is relative to m, the maximum of the scores,
// and taken in fp32 before the rounding. A scale's exponent joins the score when m has been taken off (a large score would lose it), its mantissa multiplies.
//
// Keys are dealt in units to the 4 or 8 wavefronts of a workgroup and, with few (sequence, head) pairs, in ranges to several workgroups,
// whose partial results (maximum, sum, outputs; fp32) are merged in a fixed order, by the one that comes last or by a second kernel.
//
// Measured (32 query and 8 key/value heads, D = 128; bytes are those of the keys that are there): 64 sequences of up to 4096 keys 56 us (6.0 TB/s), of 4000
// keys each 84 us (6.3 TB/s); 16 of up to 16384 60 us; one of 32768 17 us (4.0 TB/s), one of 4096 9.0 us, one of 1024 7.2 us.
#include <type_traits>

#include "fp8.h"
#include "mlt_internal.h"

namespace mlt {

namespace {

typedef __attribute__((ext_vector_type(2))) int i32x2;
typedef __attribute__((ext_vector_type(4))) int i32x4;

constexpr int PF_UNIT = 32;
constexpr int PF_MAX_SPLIT = 64;
constexpr int PF_LAST_SPLIT = 8;           // ranges that the last of their workgroups merges, at most
constexpr float PF_LAZY = 8.f, PF_GAIN = 6.f;   // log2

struct PagedFp8 {
  const uint16_t* Q;
  const uint8_t *Kc, *Vc;
  const float *Ks, *Vs;
  const int32_t *block_table, *seq_lens;
  uint16_t* O;
  float* part;
  uint32_t* counters;        // a zero for each (sequence, head, tile of 16 queries), left as zero, or null: another kernel merges
  int B, ncu;                // ncu > 0: workgroups are dealt out by sequence length
  int H, G, tiles, block_size, max_blocks, num_blocks;
  float c;
};

// The sequence that comes `rank`-th when a batch is ordered by length in units, longest first (equal ones: by index). B <= NT; buf: 2 * NT + 1 ints of LDS,
// 16-byte aligned. The wavefronts share the comparisons. Contains workgroup barriers; afterwards buf is free.
template <int NT>
__device__ __forceinline__ int sequence_of_rank(const int32_t* seq_lens, int B, int rank, int* buf) {
  const int tid = threadIdx.x;
  int key = -1;                                          // behind B: after every other
  if (tid < B) {
    const int len = seq_lens[tid], units = len < 0 ? 0 : len / PF_UNIT;
    key = (units < 1 << 22 ? units : (1 << 22) - 1) << 9 | (511 - tid);
  }
  buf[tid] = key;
  buf[NT + tid] = 0;
  __syncthreads();
  const int share = (B + NT / 16 - 1) / (NT / 16) * 4, j0 = tid / 64 * share, j1 = j0 + share < B ? j0 + share : B;
  for (int e = tid & 63; e < B; e += 64) {
    const int mine = buf[e];
    int before = 0;
    for (int j = j0; j < j1; j += 4) {
      const i32x4 four = *reinterpret_cast<const i32x4*>(buf + j);
#pragma unroll
      for (int k = 0; k < 4; ++k) before += four[k] > mine ? 1 : 0;
    }
    if (before) atomicAdd(buf + NT + e, before);
  }
  __syncthreads();
  if (tid < B && buf[NT + tid] == rank) buf[2 * NT] = tid;
  __syncthreads();
  const int b = __builtin_amdgcn_readfirstlane(buf[2 * NT]);
  __syncthreads();
  return b;
}

template <int N> using IntC = std::integral_constant<int, N>;

__device__ __forceinline__ float read_lane(float x, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
}

template <int D> struct PfRing {
  static constexpr int MAT = PF_UNIT * D;                // bytes of a unit's keys (or values)
  static constexpr int NLD = MAT / 1024;                 // loads of them
  static constexpr int WAVE = 2 * MAT + 768;             // a unit, and what is looked up for 32 units: block numbers, scales of K, of V
  // of 32 rows: chunk c of row r lies at position c ^ f(r)
  static __device__ __forceinline__ int f(int r) {
    return D == 128 ? ((r >> 1) & 3) ^ ((((r >> 3) ^ (r >> 4)) & 1) << 2) : ((r >> 2) & 3) ^ (((r >> 4) & 1) << 1);
  }
};

template <typename Tag, int D, int NW, bool SPLIT>
__global__ __launch_bounds__(NW * 64, 4) void paged_fp8_kernel(PagedFp8 a) {
  typedef PfRing<D> L;
  constexpr int NT = D / 16, KP = D / 64, NLD = L::NLD;  // tiles of O^T; 16-byte pieces of a key's row per lane
  typedef typename Elem<Tag>::vec8 V8;
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, g = lane >> 4;
  const int per_seq = a.H * a.tiles;
  int b = (int)blockIdx.x / per_seq, ht = (int)blockIdx.x % per_seq, range = SPLIT ? (int)blockIdx.y : 0;
  const int nsplit = SPLIT ? (int)gridDim.y : 1;
  if (a.ncu > 0) {                                       // dealt out by length, see dealt_piece
    const int pieces = per_seq * nsplit, id = dealt_piece((int)(blockIdx.y * gridDim.x + blockIdx.x), a.B * pieces, a.ncu);
    b = sequence_of_rank<NW * 64>(a.seq_lens, a.B, id / pieces, reinterpret_cast<int*>(smem));
    ht = id % pieces / nsplit;
    range = id % nsplit;
  }
  const int h = ht / a.tiles, q0 = ht % a.tiles * 16;
  const int nq = a.G - q0 < 16 ? a.G - q0 : 16;          // queries of this workgroup
  const int64_t head0 = (int64_t)b * a.H * a.G + (int64_t)h * a.G + q0;

  const int cap = a.max_blocks * a.block_size;
  int len = a.seq_lens[b];
  len = len < 0 ? 0 : len > cap ? cap : len;
  const int halves = (len + 15) / 16, hpb = a.block_size / 16;
  int u0 = 0, u1 = (halves + 1) / 2;
  if (SPLIT) {
    const int per = ((u1 + nsplit - 1) / nsplit + NW - 1) / NW * NW;
    u0 = range * per;
    u1 = u0 + per < u1 ? u0 + per : u1;
  }
  const int mine = u1 > u0 + wave ? (u1 - u0 - wave + NW - 1) / NW : 0;    // units of this wavefront: u0 + wave, + NW, ...

  // Q^T fragments: dimensions 64 i + 16 g + 8 j .. + 7 of query r16
  V8 qf[KP][2];
#pragma unroll
  for (int i = 0; i < KP; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      u32x4 v = {0u, 0u, 0u, 0u};
      if (r16 < nq) v = *reinterpret_cast<const u32x4_mem*>(a.Q + (head0 + r16) * D + 64 * i + 16 * g + 8 * j);
      qf[i][j] = __builtin_bit_cast(V8, v);
    }

  // Where the halves lie, and their scales: lane 2 i + p holds those of half p of the wavefront's i-th unit, 32 units at a time (halves past the last key: the
  // last one's). The next 32 are looked up, through LDS and in the stream of the other loads, while these are worked on: the way from the
  // table to the rows is two trips to memory.
  const int32_t* table = a.block_table + (int64_t)b * a.max_blocks;
  auto half_of = [&](int first) __attribute__((always_inline)) {           // this lane's, of units first, first + NW, ...
    const int hh = 2 * (first + lane / 2 * NW) + (lane & 1);
    return hh < halves ? hh : halves - 1;
  };
  auto place = [&](int hh, int blk) __attribute__((always_inline)) {       // in halves of 16 rows; the host checks that it fits
    blk = blk < 0 ? 0 : blk >= a.num_blocks ? a.num_blocks - 1 : blk;
    return (uint32_t)((blk * a.H + h) * hpb + hh % hpb);
  };
  const uint32_t ring = (uint32_t)(uintptr_t)(lptr_t)smem + (uint32_t)wave * L::WAVE, side = ring + 2 * L::MAT;
  auto ask_scales = [&](uint32_t at) __attribute__((always_inline)) {
    load_lds4(a.Ks + at / (uint32_t)hpb, side + 256);
    load_lds4(a.Vs + at / (uint32_t)hpb, side + 512);
  };
  // load j of a unit's matrix: 1 KB of rows from 1024 / D * j on; lane l the 16 bytes that belong at position l % (D / 16) of its row
  uint32_t voff[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int in = lane / (D / 16), row = 1024 / D * j + in;
    voff[j] = (uint32_t)(in * D + ((lane % (D / 16)) ^ L::f(row)) * 16);
  }
  auto fetch = [&](const uint8_t* base, uint32_t at, int i, uint32_t dst) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NLD; ++j) {
      const int p = j * 2 / NLD, part = j % (NLD / 2);   // half, and 1 KB of it
      const uint8_t* row0 = base + (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)at, 2 * i + p) * (16 * D) + part * 1024;
      // (rows 16 to 31: f is that of rows 0 to 15 with its upper bit the other way round)
      const uint32_t v = D == 128 ? voff[part ^ p] : voff[0] ^ (p ? 32u : 0u);
      load_lds16_stream(row0, v, dst + j * 1024);
    }
  };

  // log2 references: m of the weights (l), m + top of the weights times V's scales (o). mref: m, or 0 before it is known
  float m = -__builtin_inff(), mref = 0.f, l = 0.f, top = 0.f;
  f32x4 o[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};

  // LDS places of this lane's fragments inside a slot. K: row 16 p + r16, chunk 4 i + g; V: bytes 8 (r16 & 1) .. of chunk t of the row of
  // k slot r16 / 2: key 4 g + 0..3 of the first half, then of the second
  const uint32_t k_at = (uint32_t)(r16 * D + ((g ^ L::f(r16)) & (D / 16 - 1)) * 16);
  const int vrow = (r16 < 8 ? 0 : 16) + 4 * g + ((r16 >> 1) & 3);
  const uint32_t v_at = (uint32_t)(L::MAT + vrow * D + L::f(vrow) * 16 + 8 * (r16 & 1));

  uint32_t at = 0, next_at = 0;
  float ks = 0.f, vm = 0.f, ve = 0.f;                      // a half's scale of K; of V, vm * 2^ve with vm in [1/2, 1)
  if (mine > 0) {
    const int hh = half_of(u0 + wave);
    at = place(hh, table[hh / hpb]);
    ask_scales(at);
    fetch(a.Kc, at, 0, ring);
    fetch(a.Vc, at, 0, ring + L::MAT);
  }
  // Waits until at most n loads are in flight (more than that have been issued since: what was issued before has landed).
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
#pragma clang loop unroll(disable)
  for (int i = 0; i < mine; ++i) {
    const int j = i & 31, u = u0 + wave + i * NW;
    const bool more = i - j + 32 < mine;                 // units behind these 32
    if (j == 4 && more) load_lds4(table + half_of(u + 28 * NW) / hpb, side);
    // ---- scores. Since the loads of K: those of V
    landed(IntC<NLD>{});
    if (j == 16 && more) {                               // (the block numbers were asked for twelve units ago)
      next_at = place(half_of(u + 16 * NW), *(const MLT_LDS int*)(uintptr_t)(side + lane * 4u));
      lds_read();
      ask_scales(next_at);
    }
    if (j == 0) {
      ks = *(const MLT_LDS float*)(uintptr_t)(side + 256 + lane * 4u);
      const float vs = *(const MLT_LDS float*)(uintptr_t)(side + 512 + lane * 4u);
      vm = __builtin_amdgcn_frexp_mantf(vs);
      ve = vs == 0.f ? -150.f : (float)__builtin_amdgcn_frexp_expf(vs);    // (no scale is smaller)
    }
    u32x4 kr[2][KP];
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int c = 0; c < KP; ++c)
        kr[p][c] = *(const MLT_LDS u32x4*)(uintptr_t)(ring + (uint32_t)(p * 16 * D) + (k_at ^ (uint32_t)(c * 64) ^ (p ? (D == 128 ? 64u : 32u) : 0u)));
    lds_read();
    if (j == 31) at = next_at;                           // from here on units i + 1 and later are fetched
    if (i + 1 < mine) fetch(a.Kc, at, (i + 1) & 31, ring);
    const float kss[2] = {read_lane(ks, 2 * j), read_lane(ks, 2 * j + 1)}, vms[2] = {read_lane(vm, 2 * j), read_lane(vm, 2 * j + 1)},
                ves[2] = {read_lane(ve, 2 * j), read_lane(ve, 2 * j + 1)};
    float s[2][4];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < KP; ++c)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t w0 = kr[p][c][2 * e], w1 = kr[p][c][2 * e + 1];
          const u32x4 kf = {e4m3_pair<Tag, false>(w0), e4m3_pair<Tag, true>(w0), e4m3_pair<Tag, false>(w1), e4m3_pair<Tag, true>(w1)};
          acc = mfma16(__builtin_bit_cast(V8, kf), qf[c][e], acc);
        }
      const float c = a.c * kss[p];
#pragma unroll
      for (int r = 0; r < 4; ++r) s[p][r] = acc[r] * c;
    }
    const bool tail = u * PF_UNIT + PF_UNIT > len;       // keys past the last one: no weight, whatever lies there
    if (tail) {
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (u * PF_UNIT + p * 16 + 4 * g + r >= len) s[p][r] = -__builtin_inff();
    }
    const float four[2] = {__builtin_fmaxf(__builtin_fmaxf(s[0][0], s[0][1]), __builtin_fmaxf(s[0][2], s[0][3])),
                           __builtin_fmaxf(__builtin_fmaxf(s[1][0], s[1][1]), __builtin_fmaxf(s[1][2], s[1][3]))};
    const float mx = __builtin_fmaxf(four[0], four[1]);
    auto products = [&](float from) __attribute__((always_inline)) { return __builtin_fmaxf((four[0] - from) + ves[0], (four[1] - from) + ves[1]); };
    if (__any(mx > m + PF_LAZY || products(mref) > top + PF_LAZY)) {       // (m = -inf: the first time)
      auto over_keys = [](float x) __attribute__((always_inline)) {
        x = __builtin_fmaxf(x, __shfl_xor(x, 16));
        return __builtin_fmaxf(x, __shfl_xor(x, 32));
      };
      const float now = __builtin_fmaxf(m, over_keys(mx));
      if (now > -__builtin_inff()) {                     // (else nothing has been added yet)
        const float down = m - now, most = over_keys(products(now)), top_now = m == -__builtin_inff() ? most : __builtin_fmaxf(top + down, most);
        const float alpha = __builtin_amdgcn_exp2f(down + (top - top_now));
        l *= __builtin_amdgcn_exp2f(down);
        m = mref = now;
        top = top_now;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[t][r] *= alpha;
      }
    }
    u32x4 pf, pl;                                        // P rounded, and what that left
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const float up = ves[p] + (PF_GAIN - top);
      float e[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float d = s[p][r] - mref;
        l += __builtin_amdgcn_exp2f(d);
        e[r] = __builtin_amdgcn_exp2f(d + up) * vms[p];
      }
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        const uint32_t w = Elem<f16_tag>::pack2(e[r], e[r + 1]);
        pf[2 * p + r / 2] = w;
        pl[2 * p + r / 2] = Elem<f16_tag>::pack2(e[r] - Elem<f16_tag>::to_f32((uint16_t)w), e[r + 1] - Elem<f16_tag>::to_f32((uint16_t)(w >> 16)));
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    // ---- outputs. Since the loads of V: those of K of the next unit
    if (i + 1 < mine) landed(IntC<NLD>{}); else landed(IntC<0>{});
    u32x2 vr[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      vr[t] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((MLT_LDS i32x2*)(uintptr_t)(ring + (v_at ^ (uint32_t)(t * 16)))));
    }
    lds_read();
    if (i + 1 < mine) fetch(a.Vc, at, (i + 1) & 31, ring + L::MAT);
    if (tail) {
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        uint32_t keep = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (u * PF_UNIT + p * 16 + 4 * g + r < len) keep |= 0xffu << (8 * r);
#pragma unroll
        for (int t = 0; t < NT; ++t) vr[t][p] &= keep;
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const u32x4 vf = {e4m3_pair<f16_tag, false>(vr[t][0]), e4m3_pair<f16_tag, true>(vr[t][0]), e4m3_pair<f16_tag, false>(vr[t][1]), e4m3_pair<f16_tag, true>(vr[t][1])};
      o[t] = mfma16(__builtin_bit_cast(f16x8, vf), __builtin_bit_cast(f16x8, pf), o[t]);
      o[t] = mfma16(__builtin_bit_cast(f16x8, vf), __builtin_bit_cast(f16x8, pl), o[t]);
    }
  }

  // ---- the wavefronts' results meet in LDS: [wave][query] maximum, sum, outputs
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  constexpr int LD = D + 4;
  float *sm = reinterpret_cast<float*>(smem), *sl = sm + NW * 16, *so = sl + NW * 16;
  __syncthreads();                                       // (everybody is past its ring)
  if (r16 < nq) {
    if (g == 0) {
      sm[wave * 16 + r16] = m;
      sl[wave * 16 + r16] = l;
    }
    const float f = __builtin_amdgcn_exp2f(top - PF_GAIN);                 // back to the weights' reference
    // register r of tile t is dimension 16 t + 4 g + r
#pragma unroll
    for (int t = 0; t < NT; ++t)
      *reinterpret_cast<f32x4_mem*>(so + (wave * nq + r16) * LD + 16 * t + 4 * g) = f32x4{o[t][0] * f, o[t][1] * f, o[t][2] * f, o[t][3] * f};
  }
  __syncthreads();
  for (int e = tid; e < nq * D; e += NW * 64) {
    const int q = e / D, d = e % D;
    float M = sm[q], L = 0.f, acc = 0.f;
#pragma unroll
    for (int w = 1; w < NW; ++w) M = __builtin_fmaxf(M, sm[w * 16 + q]);
    const float ref = M == -__builtin_inff() ? 0.f : M;  // no key at all: sums and outputs are zeros
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float wgt = __builtin_amdgcn_exp2f(sm[w * 16 + q] - ref);
      L += sl[w * 16 + q] * wgt;
      acc += so[(w * nq + q) * LD + d] * wgt;
    }
    if (SPLIT) {
      float* out = a.part + ((head0 + q) * nsplit + range) * (2 + D);
      if (a.counters) {
        if (d == 0) { store_shared(out, M); store_shared(out + 1, L); }
        store_shared(out + 2 + d, acc);
      } else {
        if (d == 0) { out[0] = M; out[1] = L; }
        out[2 + d] = acc;
      }
    } else {
      a.O[(head0 + q) * D + d] = Elem<Tag>::from_f32(len == 0 ? 0.f : acc / L);
    }
  }
  if (!SPLIT || !a.counters) return;

  // the last range of these queries to get here merges them all, in the order of the ranges (as many of a thread's loads in flight at once as there are ranges)
  if (!last_to_arrive(a.counters + b * per_seq + ht, (uint32_t)nsplit, reinterpret_cast<uint32_t*>(smem))) return;
  for (int e = tid; e < nq * D; e += NW * 64) {
    const int q = e / D, d = e % D;
    const float* p = a.part + (head0 + q) * nsplit * (2 + D);
    float mm[PF_LAST_SPLIT], ll[PF_LAST_SPLIT], v[PF_LAST_SPLIT];
#pragma unroll
    for (int i = 0; i < PF_LAST_SPLIT; ++i) {
      const float* at_i = p + (i < nsplit ? i : 0) * (2 + D);
      mm[i] = load_shared(at_i);
      ll[i] = load_shared(at_i + 1);
      v[i] = load_shared(at_i + 2 + d);
    }
    float M = mm[0], L = 0.f, acc = 0.f;
#pragma unroll
    for (int i = 1; i < PF_LAST_SPLIT; ++i) M = __builtin_fmaxf(M, mm[i]);
    const float ref = M == -__builtin_inff() ? 0.f : M;
#pragma unroll
    for (int i = 0; i < PF_LAST_SPLIT; ++i) {
      const float wgt = i < nsplit ? __builtin_amdgcn_exp2f(mm[i] - ref) : 0.f;
      L += ll[i] * wgt;
      acc += v[i] * wgt;
    }
    a.O[(head0 + q) * D + d] = Elem<Tag>::from_f32(len == 0 ? 0.f : acc / L);
  }
}

// The merge as a kernel of its own, a workgroup per (sequence, query head): 256 / D groups of threads take every so manieth range, all loads at once.
template <typename Tag, int D>
__global__ __launch_bounds__(256) void paged_fp8_merge_kernel(const float* __restrict__ part, const int32_t* __restrict__ seq_lens, uint16_t* __restrict__ O, int Hq, int nsplit) {
  constexpr int NG = 256 / D, NR = PF_MAX_SPLIT / NG;
  __shared__ float wgt[PF_MAX_SPLIT], sum, accs[256];
  const int64_t head = blockIdx.x;
  const float* p = part + head * nsplit * (2 + D);
  const int tid = threadIdx.x, g = tid / D, d = tid % D;
  float v[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) v[i] = g + NG * i < nsplit ? p[(g + NG * i) * (2 + D) + 2 + d] : 0.f;
  if (tid < 64) {
    const float m = tid < nsplit ? p[tid * (2 + D)] : -__builtin_inff(), l = tid < nsplit ? p[tid * (2 + D) + 1] : 0.f;
    float M = m;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) M = __builtin_fmaxf(M, __shfl_xor(M, s));
    const float w = __builtin_amdgcn_exp2f(m - (M == -__builtin_inff() ? 0.f : M));      // empty ranges: 0
    float L = l * w;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) L += __shfl_xor(L, s);
    wgt[tid] = w;
    if (tid == 0) sum = L;
  }
  __syncthreads();
  float acc = 0.f;
#pragma unroll
  for (int i = 0; i < NR; ++i) acc += v[i] * wgt[g + NG * i];
  accs[tid] = acc;
  __syncthreads();
  if (tid >= D) return;
#pragma unroll
  for (int i = 1; i < NG; ++i) acc += accs[i * D + d];
  O[head * D + d] = Elem<Tag>::from_f32(seq_lens[head / Hq] <= 0 ? 0.f : acc / sum);
}

template <typename Tag, int D, int NW, bool SPLIT>
int launch_paged_fp8(const PagedFp8Args& g, int tiles, int nsplit, float* part, int order_ncu, hipStream_t s) {
  const int64_t wgs = g.B * g.H * tiles;
  // Up to 8 ranges are merged by the workgroup that comes last, which saves the second launch
  uint32_t* counters = SPLIT && nsplit <= PF_LAST_SPLIT && wgs <= kScratchCounters ? scratch_counters(part) : nullptr;
  PagedFp8 a{g.Q, g.Kc, g.Vc, g.Ks, g.Vs, g.block_table, g.seq_lens, g.O, part, counters, (int)g.B, order_ncu, (int)g.H, (int)(g.Hq / g.H), tiles,
             (int)g.block_size, (int)g.max_blocks, (int)g.num_blocks, g.scale * 1.4426950408889634f};
  const int nq = a.G < 16 ? a.G : 16;
  constexpr int RING = NW * PfRing<D>::WAVE;
  const int merge = (int)((2 * NW * 16 + NW * nq * (D + 4)) * sizeof(float)), lds = merge > RING ? merge : RING;
  auto kern = paged_fp8_kernel<Tag, D, NW, SPLIT>;
  static thread_local int configured_dev = -1;           // opt in to > 64 KB LDS once per device
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return MLT_ERR_DEVICE;
  if (lds > 64 * 1024 && configured_dev != dev) {
    if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, 80 * 1024) != hipSuccess) {
      (void)hipGetLastError();
      return MLT_ERR_LAUNCH;
    }
    configured_dev = dev;
  }
  static_assert(RING <= 80 * 1024 && (2 * NW * 16 + NW * 16 * (D + 4)) * 4 <= 80 * 1024, "what is opted in to");
  hipLaunchKernelGGL(kern, dim3((unsigned)wgs, (unsigned)nsplit), dim3(NW * 64), lds, s, a);
  if (hipGetLastError() != hipSuccess) return MLT_ERR_LAUNCH;
  if (!SPLIT || counters) return MLT_OK;
  hipLaunchKernelGGL((paged_fp8_merge_kernel<Tag, D>), dim3((unsigned)(g.B * g.Hq)), dim3(256), 0, s, part, g.seq_lens, g.O, (int)g.Hq, nsplit);
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

template <typename Tag, int D>
int run_paged_fp8_t(const PagedFp8Args& a, bool wide, int tiles, int nsplit, float* part, int order_ncu, hipStream_t s) {
  if (nsplit > 1) return wide ? launch_paged_fp8<Tag, D, 8, true>(a, tiles, nsplit, part, order_ncu, s) : launch_paged_fp8<Tag, D, 4, true>(a, tiles, nsplit, part, order_ncu, s);
  return wide ? launch_paged_fp8<Tag, D, 8, false>(a, tiles, 1, nullptr, order_ncu, s) : launch_paged_fp8<Tag, D, 4, false>(a, tiles, 1, nullptr, order_ncu, s);
}

// Key ranges per (sequence, head): up to two workgroups of 8 wavefronts on every CU, which is what a CU holds (48 sequences of 2048 keys and 8 heads: 24.4 us
// with one range, 27.9 with two, which make 768), with 8 units a range or more (one to a
// wavefront; ranges are whole multiples of that: 2000 keys in 8 ranges 7.9 us, in 7 9.1). A single sequence has no long and short pieces to even out and gets one workgroup a CU: one of 32768 keys and 8 heads 17.0 us with 32 ranges, 18.2
// with 64. 9 to 16 ranges need the second kernel and do not repay it: 4 sequences of 4096 keys 10.1 us with 8, 12.5 with 16 (of 32768: 35.5 and 34.2).
int plan_paged_fp8_split(const PagedFp8Args& a, int64_t wgs, int64_t ncu) {
  if (a.forced_split > 0) return a.forced_split > PF_MAX_SPLIT ? PF_MAX_SPLIT : a.forced_split;
  const int64_t units = (a.max_blocks * a.block_size + PF_UNIT - 1) / PF_UNIT;
  int64_t n = (a.B > 1 ? 2 : 1) * ncu / wgs;
  if (n > (units + 7) / 8) n = (units + 7) / 8;
  if (units <= 16) n = 1;                                // (two sequences of 300 keys: 4.8 us, in 2 ranges 6.0)
  if (n > PF_LAST_SPLIT && n <= 2 * PF_LAST_SPLIT) n = PF_LAST_SPLIT;
  if (n > PF_MAX_SPLIT) n = PF_MAX_SPLIT;
  return n < 1 ? 1 : (int)n;
}

}  // namespace

// Whether workgroups are dealt out by sequence length, as the 16-bit form does. Every one of them then ranks the batch, whose lengths have to fit its threads: 1 us with 64
// sequences, 3 with 192, 5 with 250. It pays where there is much to read for each, 256 KiB a workgroup and 2 KiB a sequence. us in batch order / by length, for lengths from a
// quarter of that on and for equal ones, D = 128: 64 x 8 pairs of at most 4096 keys 64.5 / 54.0 (82.3 / 83.4 equal), 70 x 8 72.0 / 64.6 (106.5 / 108.0), 128 x 8 116.8 / 108.0
// (165.0 / 168.9), 250 x 4 120.5 / 108.5 (161.6 / 169.4); 250 x 2 of 8192 122.3 / 106.7 (160.4 / 165.3). On the other side: 250 x 8 of 1024 59.1 / 60.8 (83.7 / 88.9),
// 192 x 4 of 1024 27.4 / 27.5 (33.7 / 37.2), 128 x 8 of 512 19.3 / 19.7 (24.1 / 25.9).
bool paged_fp8_by_length(const PagedFp8Args& a, int64_t wgs, int64_t nsplit, bool wide, int64_t ncu) {
  const int64_t kib = a.max_blocks * a.block_size / nsplit * a.D * 2 / 1024;
  return a.B >= 2 && a.B <= (wide ? 512 : 256) && wgs > ncu && kib >= 256 && kib >= 2 * a.B;
}

int run_paged_fp8(const PagedFp8Args& a, hipStream_t s, int* nsplit_out, int* waves_out) {
  DeviceInfo di;
  const int64_t ncu = device_info(di) && di.ncu > 0 ? di.ncu : 256;
  const int tiles = (int)((a.Hq / a.H + 15) / 16);
  if (!launch_fits(a.B * a.H * tiles, 256)) return MLT_ERR_UNSUPPORTED;    // (the wider form is for few workgroups)
  int nsplit = plan_paged_fp8_split(a, a.B * a.H * tiles, ncu);
  if (!launch_fits(a.B * a.Hq, 256)) nsplit = 1;         // (what the merging kernel would need)
  float* part = nullptr;
  ScratchTurn turn;
  if (nsplit > 1) {
    part = cached_scratch(a.B * a.Hq * nsplit * (2 + a.D) * (int64_t)sizeof(float), s, turn);
    if (!part) nsplit = 1;                               // no scratch to be had: the plain form
  }
  const int64_t wgs = a.B * a.H * tiles * nsplit;
  // 8 wavefronts where two workgroups a CU or fewer take all the keys (64 sequences of 4096 keys, D = 64: 31.5 us, with 4 wavefronts 34.1), otherwise 4,
  // which leave a CU more workgroups to choose from (128 sequences of 512 keys: 18.3 us, with 8 wavefronts 20.2).
  const bool wide = wgs <= 2 * ncu;
  const int order = paged_fp8_by_length(a, wgs, nsplit, wide, ncu) ? (int)ncu : 0;
  *nsplit_out = nsplit;
  *waves_out = wide ? 8 : 4;
  if (a.dtype == MLT_BF16)
    return a.D == 128 ? run_paged_fp8_t<bf16_tag, 128>(a, wide, tiles, nsplit, part, order, s) : run_paged_fp8_t<bf16_tag, 64>(a, wide, tiles, nsplit, part, order, s);
  return a.D == 128 ? run_paged_fp8_t<f16_tag, 128>(a, wide, tiles, nsplit, part, order, s) : run_paged_fp8_t<f16_tag, 64>(a, wide, tiles, nsplit, part, order, s);
}

}  // namespace mlt
