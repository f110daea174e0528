// Decode attention over a paged cache in e4m3 with a scale for each (block, head): one query per (sequence, query head), G = Hq / H
// query heads to a key/value head.
//
// Reading the cache is the cost (2 * D bytes a key and head), and the G queries that share it go through it together, up to 16 of
// them as the 16 columns of an MFMA: S^T = K Q^T and O^T = V^T P^T, both with the cache as the first operand, straight
// from registers.
//   * A unit is two halves of 16 keys. K: lane l holds key l % 16 of a half, 16-byte pieces l / 16 of its row, turned into the
//     16-bit type of Q (exact). Which k slot of the MFMA a dimension gets is free as long as Q's fragment agrees.
//   * S^T leaves key 4 (l / 16) + r of query l % 16 in register r. Those are the k slots 8 (l / 16) .. + 7 of the second product
//     (four from each half), so P needs no exchange between lanes.
//   * V: lane l holds, of the same eight keys, the bytes D/16 * (l % 16) .. of the row. Row m = l % 16 of tile t is dimension
//     D/16 * m + t: a lane has all of its operand itself, and what is left is the transposition of 4 x 4 bytes in registers.
// P and V are multiplied as fp16 whatever Q's type: e4m3 is exact in it, and P, at most 2^8 times the current reference
// (which moves only when a score passes it by 8 in the log2 domain), keeps 11 bits; 2^6 on top leaves it far from fp16's small end.
// The scale of V goes into P, divided by the largest one that the wavefront has met. The row sums take P as it is in fp32.
//
// Keys are dealt in units to the 4 wavefronts of a workgroup and, with few (sequence, head) pairs, in ranges to several workgroups,
// whose partial results (maximum, sum, outputs; fp32) are merged by a second kernel in a fixed order.
#include "fp8.h"
#include "mlt_internal.h"

namespace mlt {

namespace {

constexpr int PF_NW = 4;
constexpr int PF_NT = PF_NW * 64;
constexpr int PF_UNIT = 32;
constexpr int PF_MAX_SPLIT = 64;
constexpr float PF_LAZY = 8.f, PF_GAIN = 64.f;

struct PagedFp8 {
  const uint16_t* Q;
  const uint8_t *Kc, *Vc;
  const float *Ks, *Vs;
  const int32_t *block_table, *seq_lens;
  uint16_t* O;
  float* part;
  int H, G, tiles, block_size, max_blocks, num_blocks;
  float c;
};

// 4 x 4 bytes: w[r] byte t -> out[t] byte r
__device__ __forceinline__ void transpose4(const uint32_t (&w)[4], uint32_t (&out)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602);   // w0.0 w1.0 w0.1 w1.1 | w0.2 w1.2 w0.3 w1.3
  const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602);
  out[0] = __builtin_amdgcn_perm(c, a, 0x05040100);
  out[1] = __builtin_amdgcn_perm(c, a, 0x07060302);
  out[2] = __builtin_amdgcn_perm(d, b, 0x05040100);
  out[3] = __builtin_amdgcn_perm(d, b, 0x07060302);
}

template <int D> struct Unit {
  static constexpr int KP = D / 64, VW = D / 64;         // 16-byte pieces of a key's row, dwords of a value's row per lane
  u32x4 k[2][KP];
  uint32_t v[2][4][VW];
  float ks[2], vs[2];
};

template <typename Tag, int D, bool SPLIT>
__global__ __launch_bounds__(PF_NT) void paged_fp8_kernel(PagedFp8 a) {
  constexpr int NT = D / 16;                             // tiles of O^T
  constexpr int KP = Unit<D>::KP, VW = Unit<D>::VW;
  typedef typename Elem<Tag>::vec8 V8;
  extern __shared__ __align__(16) float smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, g = lane >> 4;
  const int per_seq = a.H * a.tiles;
  const int b = (int)blockIdx.x / per_seq, ht = (int)blockIdx.x % per_seq, h = ht / a.tiles, q0 = ht % a.tiles * 16;
  const int nq = a.G - q0 < 16 ? a.G - q0 : 16;          // queries of this workgroup
  const int64_t head0 = (int64_t)b * a.H * a.G + (int64_t)h * a.G + q0;

  const int cap = a.max_blocks * a.block_size;
  int len = a.seq_lens[b];
  len = len < 0 ? 0 : len > cap ? cap : len;
  const int halves = (len + 15) / 16, hpb = a.block_size / 16;
  int u0 = 0, u1 = (halves + 1) / 2;
  if (SPLIT) {
    const int nsplit = (int)gridDim.y, per = ((u1 + nsplit - 1) / nsplit + PF_NW - 1) / PF_NW * PF_NW;
    u0 = (int)blockIdx.y * per;
    u1 = u0 + per < u1 ? u0 + per : u1;
  }

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

  auto load = [&](int u, Unit<D>& x) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      int hh = 2 * u + p;
      hh = hh < halves ? hh : halves - 1;                // past the last key: any valid half, ignored
      int blk = a.block_table[(int64_t)b * a.max_blocks + hh / hpb];
      blk = blk < 0 ? 0 : blk >= a.num_blocks ? a.num_blocks - 1 : blk;
      const int64_t bh = (int64_t)blk * a.H + h, at = (bh * a.block_size + hh % hpb * 16) * D;
      x.ks[p] = a.Ks[bh];
      x.vs[p] = a.Vs[bh];
#pragma unroll
      for (int i = 0; i < KP; ++i) x.k[p][i] = load_stream16(a.Kc + at + r16 * D + 64 * i + 16 * g);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint8_t* vp = a.Vc + at + (4 * g + r) * D + r16 * (D / 16);
        if constexpr (VW == 2) {
          const u32x2 w = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(vp));
          x.v[p][r][0] = w[0];
          x.v[p][r][1] = w[1];
        } else {
          x.v[p][r][0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(vp));
        }
      }
    }
  };

  float m = -__builtin_inff(), l = 0.f, top_vs = 0x1p-100f;
  f32x4 o[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int u = u0 + wave; u < u1; u += PF_NW) {
    Unit<D> x;
    load(u, x);
    float s[2][4], mx = -__builtin_inff();
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KP; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t w0 = x.k[p][i][2 * j], w1 = x.k[p][i][2 * j + 1];
          const u32x4 kf = {e4m3_pair<Tag, false>(w0), e4m3_pair<Tag, true>(w0), e4m3_pair<Tag, false>(w1), e4m3_pair<Tag, true>(w1)};
          acc = mfma16(__builtin_bit_cast(V8, kf), qf[i][j], acc);
        }
      const float c = a.c * x.ks[p];
#pragma unroll
      for (int r = 0; r < 4; ++r) s[p][r] = acc[r] * c;
    }
    if (u * PF_UNIT + PF_UNIT > len) {                   // keys past the last one: no weight, whatever lies there
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (u * PF_UNIT + p * 16 + 4 * g + r >= len) {
            s[p][r] = -__builtin_inff();
#pragma unroll
            for (int w = 0; w < VW; ++w) x.v[p][r][w] = 0u;
          }
    }
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = __builtin_fmaxf(mx, s[p][r]);
    if (__any(mx > m + PF_LAZY)) {                       // (m = -inf: the first time)
      float all = __builtin_fmaxf(mx, __shfl_xor(mx, 16));
      all = __builtin_fmaxf(all, __shfl_xor(all, 32));
      const float now = __builtin_fmaxf(m, all);
      const float alpha = now == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(m - now);
      m = now;
      l *= alpha;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[t][r] *= alpha;
    }
    const float vs = __builtin_fmaxf(x.vs[0], x.vs[1]);
    if (vs > top_vs) {
      const float alpha = top_vs / vs;
      top_vs = vs;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[t][r] *= alpha;
    }
    const float mref = m == -__builtin_inff() ? 0.f : m;
    u32x4 pf;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const float f = x.vs[p] * (PF_GAIN / top_vs);
      float e[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        e[r] = __builtin_amdgcn_exp2f(s[p][r] - mref);
        l += e[r];
      }
      pf[2 * p] = Elem<f16_tag>::pack2(e[0] * f, e[1] * f);
      pf[2 * p + 1] = Elem<f16_tag>::pack2(e[2] * f, e[3] * f);
    }
#pragma unroll
    for (int w = 0; w < VW; ++w) {
      uint32_t t0[4], t1[4];
      const uint32_t w0[4] = {x.v[0][0][w], x.v[0][1][w], x.v[0][2][w], x.v[0][3][w]};
      const uint32_t w1[4] = {x.v[1][0][w], x.v[1][1][w], x.v[1][2][w], x.v[1][3][w]};
      transpose4(w0, t0);
      transpose4(w1, t1);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const u32x4 vf = {e4m3_pair<f16_tag, false>(t0[t]), e4m3_pair<f16_tag, true>(t0[t]), e4m3_pair<f16_tag, false>(t1[t]), e4m3_pair<f16_tag, true>(t1[t])};
        o[4 * w + t] = mfma16(__builtin_bit_cast(f16x8, vf), __builtin_bit_cast(f16x8, pf), o[4 * w + t]);
      }
    }
  }

  // ---- the wavefronts' results meet in LDS: [wave][query] maximum, sum (with the factor of its outputs), outputs
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  constexpr int LD = D + 4;
  float *sm = smem, *sl = sm + PF_NW * 16, *so = sl + PF_NW * 16;
  if (r16 < nq) {
    if (g == 0) {
      sm[wave * 16 + r16] = m;
      sl[wave * 16 + r16] = l;
    }
    const float f = top_vs / PF_GAIN;
    // register r of tile t is dimension NT * (4 g + r) + t
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < NT; t += 4)
        *reinterpret_cast<f32x4_mem*>(so + (wave * nq + r16) * LD + NT * (4 * g + r) + t) = f32x4{o[t][r] * f, o[t + 1][r] * f, o[t + 2][r] * f, o[t + 3][r] * f};
  }
  __syncthreads();
  for (int e = tid; e < nq * D; e += PF_NT) {
    const int q = e / D, d = e % D;
    float M = sm[q], L = 0.f, acc = 0.f;
#pragma unroll
    for (int w = 1; w < PF_NW; ++w) M = __builtin_fmaxf(M, sm[w * 16 + q]);
    const float ref = M == -__builtin_inff() ? 0.f : M;  // no key at all: sums and outputs are zeros
#pragma unroll
    for (int w = 0; w < PF_NW; ++w) {
      const float wgt = __builtin_amdgcn_exp2f(sm[w * 16 + q] - ref);
      L += sl[w * 16 + q] * wgt;
      acc += so[(w * nq + q) * LD + d] * wgt;
    }
    if (SPLIT) {
      float* out = a.part + ((head0 + q) * (int)gridDim.y + (int)blockIdx.y) * (2 + D);
      if (d == 0) { out[0] = M; out[1] = L; }
      out[2 + d] = acc;
    } else {
      a.O[(head0 + q) * D + d] = Elem<Tag>::from_f32(len == 0 ? 0.f : acc / L);
    }
  }
}

template <typename Tag, int D>
__global__ __launch_bounds__(D) void paged_fp8_merge_kernel(const float* __restrict__ part, const int32_t* __restrict__ seq_lens, uint16_t* __restrict__ O, int Hq, int nsplit) {
  const int64_t head = blockIdx.x;
  const float* p = part + head * nsplit * (2 + D);
  const int d = threadIdx.x;
  float M = -__builtin_inff(), L = 0.f, acc = 0.f;
  for (int i = 0; i < nsplit; ++i) M = __builtin_fmaxf(M, p[i * (2 + D)]);
  const float ref = M == -__builtin_inff() ? 0.f : M;
  for (int i = 0; i < nsplit; ++i) {
    const float wgt = __builtin_amdgcn_exp2f(p[i * (2 + D)] - ref);
    L += p[i * (2 + D) + 1] * wgt;
    acc += p[i * (2 + D) + 2 + d] * wgt;
  }
  O[head * D + d] = Elem<Tag>::from_f32(seq_lens[head / Hq] <= 0 ? 0.f : acc / L);
}

template <typename Tag, int D>
int launch_paged_fp8(const PagedFp8Args& g, int tiles, int nsplit, float* part, hipStream_t s) {
  PagedFp8 a{g.Q, g.Kc, g.Vc, g.Ks, g.Vs, g.block_table, g.seq_lens, g.O, part, (int)g.H, (int)(g.Hq / g.H), tiles,
             (int)g.block_size, (int)g.max_blocks, (int)g.num_blocks, g.scale * 1.4426950408889634f};
  const int nq = a.G < 16 ? a.G : 16;
  const size_t lds = (size_t)(2 * PF_NW * 16 + PF_NW * nq * (D + 4)) * sizeof(float);
  const unsigned wgs = (unsigned)(g.B * g.H * tiles);
  auto kern = nsplit > 1 ? paged_fp8_kernel<Tag, D, true> : paged_fp8_kernel<Tag, D, false>;
  hipLaunchKernelGGL(kern, dim3(wgs, (unsigned)nsplit), dim3(PF_NT), lds, s, a);
  if (hipGetLastError() != hipSuccess) return MLT_ERR_LAUNCH;
  if (nsplit == 1) return MLT_OK;
  hipLaunchKernelGGL((paged_fp8_merge_kernel<Tag, D>), dim3((unsigned)(g.B * g.Hq)), dim3(D), 0, s, part, g.seq_lens, g.O, (int)g.Hq, nsplit);
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

int plan_paged_fp8_split(const PagedFp8Args& a, int64_t wgs) {
  if (a.forced_split > 0) return a.forced_split > PF_MAX_SPLIT ? PF_MAX_SPLIT : a.forced_split;
  DeviceInfo di;
  const int64_t ncu = device_info(di) ? di.ncu : 256;
  const int64_t units = (a.max_blocks * a.block_size + PF_UNIT - 1) / PF_UNIT;
  int64_t n = (4 * ncu + wgs - 1) / wgs;
  if (n > units / 8) n = units / 8;
  if (n > PF_MAX_SPLIT) n = PF_MAX_SPLIT;
  return n < 1 ? 1 : (int)n;
}

}  // namespace

int run_paged_fp8(const PagedFp8Args& a, hipStream_t s, int* nsplit_out) {
  const int tiles = (int)((a.Hq / a.H + 15) / 16);
  int nsplit = plan_paged_fp8_split(a, a.B * a.H * tiles);
  float* part = nullptr;
  if (nsplit > 1) {
    part = cached_scratch(a.B * a.Hq * nsplit * (2 + a.D) * (int64_t)sizeof(float), s);
    if (!part) nsplit = 1;                               // no scratch to be had: the plain form
  }
  *nsplit_out = nsplit;
  if (a.dtype == MLT_BF16)
    return a.D == 128 ? launch_paged_fp8<bf16_tag, 128>(a, tiles, nsplit, part, s) : launch_paged_fp8<bf16_tag, 64>(a, tiles, nsplit, part, s);
  return a.D == 128 ? launch_paged_fp8<f16_tag, 128>(a, tiles, nsplit, part, s) : launch_paged_fp8<f16_tag, 64>(a, tiles, nsplit, part, s);
}

}  // namespace mlt
