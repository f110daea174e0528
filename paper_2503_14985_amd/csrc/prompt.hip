// Attention of packed sequences of different lengths, grouped heads, over packed keys or a paged cache (mlt_mha_packed_fwd, mlt_paged_attn_prompt).
//
// The products, their schedule and the LDS ring are those of mha_pp.hip: workgroup = 8 wavefronts x 32 rows, key tiles of 64, S^T = K Q^T and O^T += V^T P^T on 32x32x16 MFMAs
// with P staying in registers, two groups of wavefronts half a tile apart (one in the softmax while the other one multiplies), tiles by direct loads into five slots.
// What differs:
//   * Rows are (token, head) pairs of a key/value head's whole group, and which rows of which sequence a workgroup takes it finds out by itself from the device's offsets
//     (prompt_tile.h).
//   * A wavefront's loads of a tile are 8 neighbouring rows of K and of V. In a paged cache they lie in one block (blocks are whole multiples of 16 keys): one block
//     number for each tile, read by the scalar unit a tile ahead.
//   * A row may see no key at all: weights are taken against 0 while the maximum is -inf, and a sum of 0 gives an output of 0.
//   * A masked key's weight is 0, and 0 times a V that is not finite would be NaN. A row whose output is not finite, and to whose last tiles such a V belongs that it does not
//     see, is worked out again by itself (prompt_redo). Nothing is spent on that before it is needed but one look at the outputs, 64 multiplications an item.
//
// The largest weight of a row lies between 1 and 2^8 (the reference moves when the maximum has grown by 8): fp16 weights lose nothing but what is below 2^-25 of it.
#include <stdio.h>

#include <type_traits>

#include "prompt_tile.h"

namespace mlt {

namespace {

template <typename Tag, int D, bool CAUSAL, bool PAGED>
__device__ __forceinline__ void prompt_body(const PromptKernel& p, const PromptSeq& seq, int b, int head, int qt, uint32_t lds0) {
  typedef PaCfg<D> L;
  typedef typename Elem<Tag>::vec8 V8;
  constexpr int NKK = L::NKK, NDT = L::NDT, ROWB = L::ROWB;
  constexpr int IN8 = 8 / L::LPW;                        // rows of one load
  const PromptKeys& src = p.src;
  const PromptItems& items = p.items;
  const int64_t ldq = p.ldq, ldo = p.ldo;
  const float c = p.c;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = wave >> 2;                             // waves w and w+4 share a SIMD
  const int lq = lane & 31, h = lane >> 5;
  const int G = items.G, rows = seq.n * G, m = seq.m;
  const int q0 = qt * PA_BM + wave * 32;                 // first row of this wavefront
  const int my_r = q0 + lq, last_r = rows - 1;
  const int my_tok = (my_r < last_r ? my_r : last_r) / G;   // (rows past the last one repeat it and are not stored)

  // Keys that row r sees: those before end(r) (all of them without the mask), none where that is 0 or less.
  const int shift = m - seq.n + 1;
  auto end_of = [&](int r) { return CAUSAL ? shift + uniform((r < last_r ? r : last_r) / G) : m; };
  const int wg_end = end_of((qt + 1) * PA_BM - 1), w_first = end_of(q0), w_end = end_of(q0 + 31), my_end = CAUSAL ? shift + my_tok : m;
  const int my_last = my_end - 1 - 4 * h;                // ... from the first key that this lane holds of 8
  const int nblk = wg_end > 0 ? (wg_end + PA_BN - 1) / PA_BN : 0;
  // This wavefront has visible keys in tiles 0 .. my_nblk-1 only.
  const int my_nblk = w_end > 0 && q0 < rows ? (w_end + PA_BN - 1) / PA_BN : 0;

  V8 qf[NKK];                                            // Q^T operand: row lq, d = 16*kk + 8*h .. +7

  // ---- global -> LDS assignments: wavefront w fills rows 8 w .. 8 w + 7 of the K tile and of the V tile; lane l owns the 16-byte slot l of a 1 KB block.
  const uint32_t rowk = PAGED ? ROWB : (uint32_t)src.ldk * 2, rowv = PAGED ? ROWB : (uint32_t)src.ldv * 2;
  uint32_t voff_k[L::LPW], voff_v[L::LPW];               // byte offsets from the first of the 8 rows, all of them there
  // `have`: rows behind the first one that are there; those past them re-read the last one (their weights are 0)
  auto offsets_of = [&](int ln, int i, int have, uint32_t& ok, uint32_t& ov) __attribute__((always_inline)) {
    const int in8 = i * IN8 + ln / L::CPR, slot = ln % L::CPR, at = in8 < have ? in8 : have;
    ok = (uint32_t)at * rowk + (uint32_t)(slot ^ L::fk(wave * 8 + in8)) * 16u;
    ov = (uint32_t)at * rowv + (uint32_t)(slot ^ L::fv(wave * 8 + in8)) * 16u;
  };
#pragma unroll
  for (int i = 0; i < L::LPW; ++i) offsets_of(lane, i, 7, voff_k[i], voff_v[i]);
  const int last_key = wg_end - 1;                       // of what this workgroup reads
  PromptCursor<D, 8, PAGED> at;                          // (K and V of a packed sequence may have other strides: ...)
  auto first_tile = [&]() __attribute__((always_inline)) { at.start(src, src.K, src.ldk, seq, b, items.H, head, last_key, wave * 8, PA_BN); };
  auto issue_tile = [&](int t) __attribute__((always_inline)) {
    const uint32_t dst = lds0 + (t % PA_NS) * L::SLOT_B + wave * L::LPW * 1024;
    int have;
    const int key = at.key < last_key ? at.key : last_key;
    const char* kp = at.next(have);
    const char* vp = uniform(PAGED ? reinterpret_cast<const char*>(src.V) + (kp - reinterpret_cast<const char*>(src.K))
                                   : reinterpret_cast<const char*>(src.V + (int64_t)(seq.k0 + key) * src.ldv + (int64_t)head * D));   // (... this is V's)
    if (D == 128 && have == 7) {                         // (D = 64 has no registers to keep them in)
#pragma unroll
      for (int i = 0; i < L::LPW; ++i) load_lds16(kp, voff_k[i], dst + i * 1024);
#pragma unroll
      for (int i = 0; i < L::LPW; ++i) load_lds16(vp, voff_v[i], dst + L::TILE_B + i * 1024);
    } else {
      int ln = lane;
      asm volatile("" : "+v"(ln));
#pragma unroll
      for (int i = 0; i < L::LPW; ++i) {
        uint32_t ok, ov;
        offsets_of(ln, i, have, ok, ov);
        load_lds16(kp, ok, dst + i * 1024);
        load_lds16(vp, ov, dst + L::TILE_B + i * 1024);
      }
    }
  };

  f32x16 o_acc[NDT];
  f32x16 s_acc[2];
  u32x4 pq[4];                       // P^T of the current tile as MFMA operands: one per 16 keys
  float mc_run, l_run;
  V8 fb[2][NDT];
  // Fragment addresses: one per XOR variant in a register, moved from slot to slot; D = 64, which has no registers to spare, keeps one of K's and works out the others
  constexpr int NKA = D == 64 ? 1 : NKK;
  uint32_t ka[NKA], va[NDT];
  auto read_v_frag = [&](int g, int t, V8& f) {
    const uint32_t a = va[t] + g * 16 * ROWB;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((MLT_LDS s16x4*)(uintptr_t)a);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((MLT_LDS s16x4*)(uintptr_t)(a + 8 * ROWB));
    f = join_tr<V8>(lo, hi);
  };
  auto read_k_frag = [&](int fi, V8& f) {
    const uint32_t a = (NKA == 1 ? ka[0] ^ ((fi >> 1) << 5) : ka[(fi >> 1) % NKA]) + (fi & 1) * 32 * ROWB;
    f = __builtin_bit_cast(V8, *(const MLT_LDS u32x4*)(uintptr_t)a);
  };
  auto mfma_v = [&](int g, int t, const V8& f) { o_acc[t] = mfma32(f, __builtin_bit_cast(V8, pq[g]), o_acc[t]); };
  auto mfma_k = [&](int fi, const V8& f) {
    if (fi < 2) {
      f32x16 z;
#pragma unroll
      for (int r = 0; r < 16; ++r) z[r] = 0.f;
      s_acc[fi & 1] = mfma32(f, qf[fi >> 1], z);
    } else {
      s_acc[fi & 1] = mfma32(f, qf[fi >> 1], s_acc[fi & 1]);
    }
  };
#define MLT_SB() __builtin_amdgcn_sched_barrier(0)
  auto cut = [&](int j) { return (j + 1) * PA_BN > w_first; };         // does the mask, or the last key, cut tile j for this wavefront?

  // ---- softmax of S_j (in s_acc) -> pq, mc_run, rescaled o_acc and l_run (see mha_pp_kernel)
  auto softmax_tile = [&](int j) {
    // register r of sub-tile kb is key 64 j + 32 kb + 8 (r / 4) + 4 h + r % 4
    if (cut(j)) {
      const int rel = my_last - j * PA_BN;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * kb + 8 * (r >> 2) + (r & 3) > rel) s_acc[kb][r] = -__builtin_inff();
    }
    float mx = max3(s_acc[0][0], s_acc[0][1], s_acc[0][2]);
#pragma unroll
    for (int r = 3; r < 15; r += 2) mx = max3(mx, s_acc[0][r], s_acc[0][r + 1]);
    mx = max3(mx, s_acc[0][15], s_acc[1][0]);
#pragma unroll
    for (int r = 1; r < 15; r += 2) mx = max3(mx, s_acc[1][r], s_acc[1][r + 1]);
    mx = __builtin_fmaxf(mx, s_acc[1][15]);
    mx = both_halves_max(mx);
    const float t = mx * c;
    const bool grow = t - mc_run > PA_LAZY_T;
    if (__builtin_amdgcn_ballot_w64(grow) != 0) {
      const float alpha = grow ? __builtin_amdgcn_exp2f(mc_run - t) : 1.f;
      l_run *= alpha;
#pragma unroll
      for (int tt = 0; tt < NDT; ++tt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o_acc[tt][r] *= alpha;
      mc_run = grow ? t : mc_run;
    }
    const float ref = mc_run == -__builtin_inff() ? 0.f : mc_run;        // (no key seen yet: all weights are exp2(-inf))
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s_acc[kb][r], c, -ref));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s_acc[kb][r + 1], c, -ref));
        pq[2 * kb + r / 8][(r / 2) & 3] = Elem<Tag>::pack2(p0, p1);
      }
  };
  constexpr int LPT = 2 * L::LPW;                         // loads per wavefront per tile
#pragma unroll
  for (int t = 0; t < NDT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) o_acc[t][r] = 0.f;
  mc_run = -__builtin_inff();    // reference point of the weights: a running maximum of the scores, times c (log2 domain)
  l_run = 0.f;                   // running sum over this lane's half of the keys
  {
    // Q, and fragment addresses inside a slot (see mha_pp_kernel), from an opaque lane number: not to be kept in registers for a second turn
    int ln = lane;
    asm volatile("" : "+v"(ln));
    const int fq = ln & 31, fh = ln >> 5;
    const int row = q0 + fq < last_r ? q0 + fq : last_r, tok = row / G;
    const uint16_t* qp = p.Q + (int64_t)(seq.q0 + tok) * ldq + (int64_t)(head * G + row - tok * G) * D + 8 * fh;
    const uint32_t flip = p.negate ? 0x80008000u : 0u;       // a negative scale as a sign flip
#pragma unroll
    for (int kk = 0; kk < NKK; ++kk) {
      u32x4 raw = *reinterpret_cast<const u32x4_mem*>(qp + kk * 16);
      raw[0] ^= flip; raw[1] ^= flip; raw[2] ^= flip; raw[3] ^= flip;
      qf[kk] = __builtin_bit_cast(V8, raw);
    }
    const int k_frag = fq * ROWB + ((fh ^ L::fk(fq)) << 4);
    const int vg = ln >> 4, vs = ln & 15;
    const int v_row = 4 * (vg >> 1) + (vs >> 2);
    const int v_frag = L::TILE_B + v_row * ROWB + (((2 * (vg & 1) + ((vs & 3) >> 1)) ^ L::fv(v_row)) << 4) + 8 * (vs & 1);
#pragma unroll
    for (int kk = 0; kk < NKA; ++kk) ka[kk] = lds0 + (uint32_t)(k_frag ^ (kk << 5));
#pragma unroll
    for (int t = 0; t < NDT; ++t) va[t] = lds0 + (uint32_t)(v_frag ^ (t << 6));
  }

  // ---- schedule: see mha_pp_kernel
  first_tile();
#pragma unroll
  for (int t = 0; t < PA_AHEAD; ++t)
    if (t < nblk) issue_tile(t);
  if (nblk >= 3) __builtin_amdgcn_s_waitcnt(wait_imm(2 * LPT, 15));
  else if (nblk == 2) __builtin_amdgcn_s_waitcnt(wait_imm(LPT, 15));
  else __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));
  MLT_BARRIER();
  if (grp == 1) MLT_BARRIER();            // stagger: group 1 runs one phase behind
  {
    if (my_nblk > 0) {                                    // ka, va point into slot 0
#pragma unroll
      for (int i = 0; i < NDT; ++i) read_k_frag(i, fb[0][i]);
#pragma unroll
      for (int i = 0; i < NDT; ++i) read_k_frag(NDT + i, fb[1][i]);
      MLT_SB();
#pragma unroll
      for (int ch = 0; ch < 4; ++ch)
#pragma unroll
        for (int i = 0; i < NDT; ++i) {
          mfma_k(ch * NDT + i, fb[ch & 1][i]);
          MLT_SB();
          if (ch < 2) read_k_frag((ch + 2) * NDT + i, fb[ch & 1][i]);
          else read_v_frag(ch - 2, i, fb[ch & 1][i]);
          MLT_SB();
        }
    }
    if (grp == 1) {
      if (nblk >= 3) __builtin_amdgcn_s_waitcnt(wait_imm(LPT, 15));
      else __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));
    }
    MLT_BARRIER();
  }

  int slot_off = 0;                                       // byte offset of tile j's slot
  for (int j = 0; j < nblk; ++j) {
    const int slot_off_next = slot_off + L::SLOT_B == L::SMEM ? 0 : slot_off + L::SLOT_B;
    const bool active = j < my_nblk;                       // wavefront-uniform
    const bool active_next = j + 1 < my_nblk;
    // ---- X_j (the first two V_j groups are already in the chunk buffers)
    if (j + PA_AHEAD < nblk) issue_tile(j + PA_AHEAD);
    __builtin_amdgcn_sched_barrier(0);
    if (active) {
      softmax_tile(j);
#pragma unroll
      for (int g = 0; g < 4; ++g) asm volatile("" : "+v"(pq[g]));
    }
    __builtin_amdgcn_sched_barrier(0);
    if (grp == 0) {
      const int newer = (j + 3 < nblk ? 1 : 0) + (j + 2 < nblk ? 1 : 0);
      if (newer == 2) __builtin_amdgcn_s_waitcnt(wait_imm(2 * LPT, 0));
      else if (newer == 1) __builtin_amdgcn_s_waitcnt(wait_imm(LPT, 0));
      else __builtin_amdgcn_s_waitcnt(wait_imm(0, 0));
    } else {
      __builtin_amdgcn_s_waitcnt(wait_imm(63, 0));
    }
    MLT_BARRIER();
    __builtin_amdgcn_sched_barrier(0);
    if (D == 128) __builtin_amdgcn_s_setprio(1);
    // ---- C_j
    if (active) {
      const uint32_t dslot = (uint32_t)(slot_off_next - slot_off);
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int t = 0; t < NDT; ++t) {
          mfma_v(g, t, fb[g & 1][t]);
          MLT_SB();
          if (g < 2) read_v_frag(g + 2, t, fb[g & 1][t]);
          else read_k_frag((g - 2) * NDT + t, fb[g & 1][t]);
          if (g == 0 && NKA > 1) { ka[(2 * t) % NKA] += dslot; ka[(2 * t + 1) % NKA] += dslot; }
          if (g == 0 && NKA == 1 && t == 0) ka[0] += dslot;
          if (g == 3) va[t] += dslot;
          MLT_SB();
        }
      if (active_next) {
#pragma unroll
        for (int ch = 0; ch < 4; ++ch)
#pragma unroll
          for (int i = 0; i < NDT; ++i) {
            mfma_k(ch * NDT + i, fb[ch & 1][i]);
            MLT_SB();
            if (ch < 2) read_k_frag((ch + 2) * NDT + i, fb[ch & 1][i]);
            else read_v_frag(ch - 2, i, fb[ch & 1][i]);
            MLT_SB();
          }
      }
      // the sum of the ROUNDED weights (what P V used), while the matrix pipe drains
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) l_run = Elem<Tag>::add_pair(pq[g][e], l_run);
      asm volatile("" : "+v"(l_run));
    }
    if (D == 128) __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
    if (grp == 1) {
      if (j + 3 < nblk) __builtin_amdgcn_s_waitcnt(wait_imm(LPT, 15));
      else __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));
    }
    MLT_BARRIER();
    __builtin_amdgcn_sched_barrier(0);
    slot_off = slot_off_next;
  }
  if (grp == 0) MLT_BARRIER();            // same barrier count for both groups


  // ---- rows to be done again: an output is not finite, and so is a value that the row's last tiles hold without its seeing it
  float sum = 0.f;                          // x * 0 is 0, or NaN where x is not finite
#pragma unroll
  for (int t = 0; t < NDT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) sum = __builtin_fmaf(o_acc[t][r], 0.f, sum);
  const uint64_t bad = __builtin_amdgcn_ballot_w64(!(sum == 0.f));
  uint32_t redo = 0;
  if (bad) redo = prompt_redo<Tag, D, CAUSAL, PAGED>(p, seq, b, head, q0, (uint32_t)bad | (uint32_t)(bad >> 32), my_nblk * PA_BN, wg_end);
#undef MLT_SB

  // ---- epilogue: O = O^T / l, l summed over both key halves, rows without keys 0; whole rows through LDS, 16 bytes a lane
  const float l_tot = both_halves_sum(l_run);
  const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
  u32x4 ow[NDT][2];
#pragma unroll
  for (int t = 0; t < NDT; ++t)
#pragma unroll
    for (int gp = 0; gp < 2; ++gp) ow[t][gp] = o_piece16<Tag>(o_acc[t], 2 * gp, inv);
  const uint32_t o_lds = lds0 + wave * 32 * ROWB;
  constexpr int CM = L::CPR - 1;
#pragma unroll
  for (int t = 0; t < NDT; ++t)
#pragma unroll
    for (int gp = 0; gp < 2; ++gp) {
      const int ch = 4 * t + 2 * gp + h;
      *(MLT_LDS u32x4*)(uintptr_t)(o_lds + lq * ROWB + ((ch ^ (lq & CM)) << 4)) = ow[t][gp];
    }
  // where row lq goes, in 16-byte pieces from the wavefront's first token on (a store writes whole rows and asks the lane that knows). Worked out again rather than kept in
  // registers through the loop.
  int ln = lane;
  asm volatile("" : "+v"(ln));
  const int out_row = q0 + (ln & 31) < last_r ? q0 + (ln & 31) : last_r, out_tok = out_row / G, tok0 = uniform((q0 < last_r ? q0 : last_r) / G);
  const int o_piece = (int)(((out_tok - tok0) * ldo + (int64_t)(out_row - out_tok * G) * D) / 8);
  uint16_t* ob = p.O + (int64_t)(seq.q0 + tok0) * ldo + (int64_t)head * G * D;
#pragma unroll
  for (int i = 0; i < 32 / L::RPB; ++i) {
    const int r = i * L::RPB + lane / L::CPR, cc = lane % L::CPR;
    const u32x4 v = *(const MLT_LDS u32x4*)(uintptr_t)(o_lds + r * ROWB + ((cc ^ (r & CM)) << 4));
    const int piece = __shfl(o_piece, r);
    if (q0 + r < rows && !(redo >> r & 1)) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_mem*>(ob + ((int64_t)piece + cc) * 8));
  }
}

template <typename Tag, int D, bool CAUSAL, bool PAGED>
__global__ __launch_bounds__(PA_NT, D == 64 ? 4 : 1) void prompt_kernel(PromptKernel p) {
  extern __shared__ __align__(16) char smem[];
  PromptSeq seq;
  int b, head, qt;
  if (!prompt_item<PA_BM, PA_NT>(p.items, reinterpret_cast<int*>(smem), seq, b, head, qt)) return;
  seq.q0 = uniform(seq.q0); seq.n = uniform(seq.n); seq.k0 = uniform(seq.k0); seq.m = uniform(seq.m);
  b = uniform(b); head = uniform(head); qt = uniform(qt);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lptr_t)smem;
  prompt_body<Tag, D, CAUSAL, PAGED>(p, seq, b, head, qt, lds0);
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
