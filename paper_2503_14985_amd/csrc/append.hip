// Appending new tokens to a paged cache: queries and keys turned by their positions' angles, keys and values written to the slots
// that the block table names, as 16-bit rows or as e4m3 with a scale for each (block, head).
//
// A token's position is its place from the end of its sequence: seq_lens counts the new tokens, and offsets[b] ..
// offsets[b + 1] - 1 are the rows of sequence b. The rotation is computed as written, product by product in fp32 and with no
// fused multiply-add, so that what is rounded afterwards does not depend on how the compiler joins them.
//
// Two kinds of wavefronts in one launch (blockIdx.x below or from `row_blocks` on):
//   * rows: one token (or a part of its heads): the token's sequence is found by a 64-way search over the offsets, its cosines and sines are loaded once into
//     registers, and its heads (query rows; in a 16-bit cache key and value rows as well) go through 16 bytes a lane.
//   * units (8-bit cache): one (cache block, head) of the keys or of the values that new tokens fall in. The scale belongs to all
//     of the block's tokens, so one owner sees all of them: the maximum over the new ones, the scale that is there if the
//     block has earlier ones, and only where that has to grow are the earlier ones read, multiplied by old / new and
//     rounded again.
// Bound by memory where there are many tokens: rows in, rows out. With few it is the chain of loads in front of the first
// store: offsets, length, block number and angles.
// Measured (32 + 8 + 8 heads of 128): 8191 tokens of 13 sequences into an 8-bit cache 36.8 us, 189 MB at 5.1 TB/s, the rate of a plain copy; a token each for 64
// sequences 4.6 us, a launch and that chain. Two heads to a wavefront (half the chains, twice the loads in flight) 35.2 us with many tokens, but 10.9 instead of
// 8.5 with 1000. The vector units are busy for a third of the time.
#include <type_traits>

#include "fp8.h"
#include "mlt_internal.h"

namespace mlt {

namespace {

// threads of a workgroup whose units have W wavefronts: 4 units of one wavefront, or one unit
constexpr int ap_threads(int W) { return W == 1 ? 256 : 64 * W; }

// The largest b of [0, B) with start(b) <= i, or -1, by all 64 lanes together; start(b) does not fall with b.
template <typename F>
__device__ __forceinline__ int find_sequence(F&& start, int B, int i, int lane) {
  int lo = 0, n = B;
  while (true) {
    const int step = n > 64 ? (n + 63) / 64 : 1, at = lane * step;
    const int count = __popcll(__ballot(at < n && start(lo + at) <= i));
    if (count == 0) return -1;
    lo += (count - 1) * step;
    if (step == 1) return lo;
    n = n - (count - 1) * step < step ? n - (count - 1) * step : step;
  }
}

// The angle of a lane's 8 elements (d = 8 c .. 8 c + 7 of the head): halves (i, i + r/2) or neighbours (2 i, 2 i + 1) are a pair.
struct Angles { float co[8], si[8]; };

template <bool NEIGHBOURS>
__device__ __forceinline__ void load_angles(Angles& a, const float* cos, const float* sin, int half, int c) {
  constexpr int N = NEIGHBOURS ? 4 : 8;
  const int i0 = NEIGHBOURS ? 4 * c : 8 * c < half ? 8 * c : 8 * c - half;
#pragma unroll
  for (int e = 0; e < N; e += 4) {
    const f32x4 x = *reinterpret_cast<const f32x4_mem4*>(cos + i0 + e), y = *reinterpret_cast<const f32x4_mem4*>(sin + i0 + e);
#pragma unroll
    for (int j = 0; j < 4; ++j) { a.co[e + j] = x[j]; a.si[e + j] = y[j]; }
  }
}

// x: the lane's 8 elements, p: those of the lane that holds the other halves (NEIGHBOURS: unused); first: x is a first half.
template <bool NEIGHBOURS>
__device__ __forceinline__ void rotate8(float (&x)[8], const float (&p)[8], const Angles& a, bool first) {
#pragma clang fp contract(off)
  if (NEIGHBOURS) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x1 = x[2 * i], x2 = x[2 * i + 1];
      const float u = x1 * a.co[i], v = x2 * a.si[i], w = x2 * a.co[i], z = x1 * a.si[i];
      x[2 * i] = u - v;
      x[2 * i + 1] = w + z;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float u = x[e] * a.co[e], v = p[e] * a.si[e];
      x[e] = first ? u - v : u + v;
    }
  }
}

// What a wavefront of either kind knows of the call
struct Append {
  int T, B, Hq, H, block_size, max_blocks, num_blocks, half, positions, row_blocks, parts, dense_items;
  const uint16_t* Q; int64_t ldq;
  const uint16_t* K; int64_t ldk;
  const uint16_t* V; int64_t ldv;
  const int32_t *offsets, *seq_lens, *block_table;
  const float *cos, *sin;
  uint16_t* Qo;
  void *Kc, *Vc;
  float *Ks, *Vs;
};

// The lane's piece of a row, turned where it lies in the rotated part; all lanes of the row call it.
template <typename Tag, int D, bool NEIGHBOURS>
__device__ __forceinline__ void turned(const u32x4& v, float (&x)[8], const Angles& a, int half, int c, int lane) {
  unpack8<Tag>(v, x);
  if (half == 0) return;
  float p[8] = {};
  const int hc = half >> 3;                              // lanes of a half
  if (!NEIGHBOURS) {
    const int from = lane + (c < hc ? hc : c < 2 * hc ? -hc : 0);
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)__shfl((int)v[i], from);
    unpack8<Tag>(w, p);
  }
  if (c < 2 * hc) rotate8<NEIGHBOURS>(x, p, a, c < hc);
}

template <typename Tag>
__device__ __forceinline__ u32x4 pack8(const float (&x)[8]) {
  return u32x4{Elem<Tag>::pack2(x[0], x[1]), Elem<Tag>::pack2(x[2], x[3]), Elem<Tag>::pack2(x[4], x[5]), Elem<Tag>::pack2(x[6], x[7])};
}

template <typename Tag, int D, bool FP8, bool NEIGHBOURS, int W>
__device__ __forceinline__ void append_rows(const Append& a, int lane, int wave) {
  constexpr int LPR = D / 8, RPI = 64 / LPR;             // lanes per row, rows per access
  const int w = (int)blockIdx.x * (ap_threads(W) / 64) + wave;
  const int t = w / a.parts, part = w % a.parts;
  if (t >= a.T) return;
  const int b = find_sequence([&](int j) { return a.offsets[j]; }, a.B, t, lane);
  if (b < 0 || t >= a.offsets[b + 1]) return;            // a row that belongs to no sequence
  const int pos = a.seq_lens[b] - a.offsets[b + 1] + t;
  const int c = lane % LPR, g = lane / LPR;
  Angles ang;
  if (a.half && 8 * c < 2 * a.half) {
    const int at = pos < 0 ? 0 : pos < a.positions ? pos : a.positions - 1;
    load_angles<NEIGHBOURS>(ang, a.cos + (int64_t)at * a.half, a.sin + (int64_t)at * a.half, a.half, c);
  }
  int64_t slot = -1;                                     // of head 0 in a 16-bit cache
  if (!FP8 && pos >= 0 && pos < a.max_blocks * a.block_size) {
    const int blk = a.block_table[(int64_t)b * a.max_blocks + pos / a.block_size];
    if (blk >= 0 && blk < a.num_blocks) slot = ((int64_t)blk * a.H * a.block_size + pos % a.block_size) * D;
  }
  const int rows = FP8 ? a.Hq : a.Hq + 2 * a.H;
  const int64_t head_stride = (int64_t)a.block_size * D;
  auto run = [&](auto several) __attribute__((always_inline)) {
    constexpr int U = decltype(several)::value;          // accesses in flight; past the last row: the last one again
    for (int r0 = part * RPI + g; r0 - g < rows; r0 += U * RPI * a.parts) {
      u32x4 v[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int r = r0 + i * RPI * a.parts < rows ? r0 + i * RPI * a.parts : rows - 1;
        const uint16_t* src = a.Q + (int64_t)t * a.ldq + r * D;
        if (!FP8) {
          const uint16_t *k = a.K + (int64_t)t * a.ldk + (r - a.Hq) * D, *v = a.V + (int64_t)t * a.ldv + (r - a.Hq - a.H) * D;
          src = r < a.Hq ? src : r < a.Hq + a.H ? k : v;
        }
        v[i] = load_stream16(src + 8 * c);
      }
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int r = r0 + i * RPI * a.parts;
        const bool plain = !FP8 && r >= a.Hq + a.H;
        float x[8];
        turned<Tag, D, NEIGHBOURS>(v[i], x, ang, a.half, c, lane);
        const u32x4 y = plain ? v[i] : pack8<Tag>(x);
        if (r < a.Hq) {
          *reinterpret_cast<u32x4_mem*>(a.Qo + ((int64_t)t * a.Hq + r) * D + 8 * c) = y;
        } else if (!FP8 && r < rows && slot >= 0) {
          uint16_t* dst = (uint16_t*)(plain ? a.Vc : a.Kc) + slot + (r - a.Hq - (plain ? a.H : 0)) * head_stride;
          *reinterpret_cast<u32x4_mem*>(dst + 8 * c) = y;
        }
      }
    }
  };
  // Four accesses at once pay where there are four of them: 8191 tokens of 32 + 8 + 8 heads of 128 into an 8-bit cache 36.8 us, one by one 38.3 (into a 16-bit one 37.0 and
  // 38.8); of 64, where a token has half the bytes, 22.6 and 21.9
  if (D == 128 && a.parts == 1 && rows >= 4 * RPI) run(std::integral_constant<int, 4>{});
  else run(std::integral_constant<int, 1>{});
}

// W wavefronts share a unit
template <typename Tag, int D, bool NEIGHBOURS, int W>
__device__ __forceinline__ void append_unit(const Append& a, int lane, int wave, float* lds) {
  constexpr int LPR = D / 8, RPI = 64 / LPR;
  constexpr int KEEP = 16 / RPI;                         // accesses whose rows stay in registers: 16 tokens
  const int upi = 2 * a.H;                               // units of an item
  const int u = ((int)blockIdx.x - a.row_blocks) * (ap_threads(W) / 64 / W) + (W == 1 ? wave : 0);
  const int item = u / upi, hk = u % upi, sub = W == 1 ? 0 : wave;
  // item -> sequence and the block of it that new tokens fall in (touched blocks of b: at most its new tokens, and at most new / block_size + 2)
  const bool dense = a.dense_items != 0;
  auto start_of = [&](int j) { return dense ? a.offsets[j] : a.offsets[j] / a.block_size + 2 * j; };
  const int b = find_sequence(start_of, a.B, item, lane);
  if (b < 0) return;
  const int o0 = a.offsets[b], o1 = a.offsets[b + 1], end = a.seq_lens[b], begin = end - (o1 - o0);
  const int from = begin < 0 ? 0 : begin;
  const int lb = from / a.block_size + item - start_of(b);
  if (lb < 0 || lb >= a.max_blocks) return;
  const int first = from > lb * a.block_size ? from : lb * a.block_size;
  const int last = (lb + 1) * a.block_size < end ? (lb + 1) * a.block_size : end;     // positions first .. last - 1
  if (first >= last) return;
  const int blk = a.block_table[(int64_t)b * a.max_blocks + lb];
  if (blk < 0 || blk >= a.num_blocks) return;
  const bool keys = hk < a.H;
  const int h = keys ? hk : hk - a.H, c = lane % LPR, g = lane / LPR;
  const uint16_t* src = keys ? a.K + h * D : a.V + h * D;
  const int64_t ld = keys ? a.ldk : a.ldv;
  uint8_t* dst = (uint8_t*)(keys ? a.Kc : a.Vc) + ((int64_t)blk * a.H + h) * a.block_size * D;   // slot 0
  float* scale_at = (keys ? a.Ks : a.Vs) + (int64_t)blk * a.H + h;
  const int slot0 = first - lb * a.block_size, n = last - first;
  const float old = slot0 > 0 ? *scale_at : 0.f;         // 0: the block held nothing of this sequence
  const int half = keys ? a.half : 0;

  // rows i of this unit (0 .. n - 1) that this access of this wavefront holds
  auto load = [&](int i, float (&x)[8]) __attribute__((always_inline)) {
    const int t = first - begin + i + o0, pos = first + i;
    const bool in = i < n && t >= 0 && t < a.T;
    u32x4 v = {0u, 0u, 0u, 0u};
    if (in) v = load_stream16(src + (int64_t)t * ld + 8 * c);
    Angles ang;
    if (half && 8 * c < 2 * half) {
      const int at = pos < a.positions ? pos : a.positions - 1;
      load_angles<NEIGHBOURS>(ang, a.cos + (int64_t)at * half, a.sin + (int64_t)at * half, half, c);
    }
    turned<Tag, D, NEIGHBOURS>(v, x, ang, half, c, lane);
    return in;
  };
  float x[KEEP][8], top = 0.f;
  bool in[KEEP];
#pragma unroll
  for (int k = 0; k < KEEP; ++k) {
    in[k] = load((k * W + sub) * RPI + g, x[k]);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = __builtin_fmaxf(top, finite_abs(x[k][e]));
  }
  for (int i0 = (KEEP * W + sub) * RPI; i0 < n; i0 += W * RPI) {
    float y[8];
    load(i0 + g, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = __builtin_fmaxf(top, finite_abs(y[e]));
  }
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, m));
  if (W > 1) {
    if (lane == 0) lds[wave] = top;
    __syncthreads();                                     // (every wavefront of the workgroup is on the same unit, and has read `old`)
#pragma unroll
    for (int i = 0; i < W; ++i) top = __builtin_fmaxf(top, lds[i]);
  }
  float s = pow2_scale(top);
  if (slot0 > 0) s = __builtin_fmaxf(s, pow2_ceil(old));
  const float inv = pow2_inv(s);
  auto store = [&](int i, const float (&y)[8]) __attribute__((always_inline)) {
    *reinterpret_cast<u32x2_mem*>(dst + (int64_t)(slot0 + i) * D + 8 * c) =
        u32x2{to_e4m3x4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv), to_e4m3x4(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv)};
  };
#pragma unroll
  for (int k = 0; k < KEEP; ++k)
    if (in[k]) store((k * W + sub) * RPI + g, x[k]);
  for (int i0 = (KEEP * W + sub) * RPI; i0 < n; i0 += W * RPI) {
    float y[8];
    if (load(i0 + g, y)) store(i0 + g, y);
  }
  if (slot0 > 0 && s != old) {                           // the earlier tokens of the block, in the new scale; eight accesses at once
    const float f = old * inv;
    for (int i0 = sub * RPI + g; i0 < slot0; i0 += 8 * W * RPI) {
      u32x2 v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int i = i0 + k * W * RPI < slot0 ? i0 + k * W * RPI : i0;
        v[k] = *reinterpret_cast<const u32x2_mem*>(dst + (int64_t)i * D + 8 * c);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int i = i0 + k * W * RPI;
        const f32x4 lo = from_e4m3x4(v[k][0]), hi = from_e4m3x4(v[k][1]);
        if (i < slot0)
          *reinterpret_cast<u32x2_mem*>(dst + (int64_t)i * D + 8 * c) =
              u32x2{to_e4m3x4(lo[0] * f, lo[1] * f, lo[2] * f, lo[3] * f), to_e4m3x4(hi[0] * f, hi[1] * f, hi[2] * f, hi[3] * f)};
      }
    }
  }
  if (sub == 0 && lane == 0 && s != old) *scale_at = s;
}

template <typename Tag, int D, bool FP8, bool NEIGHBOURS, int W>
__global__ __launch_bounds__(ap_threads(W)) void append_kernel(Append a) {
  __shared__ float lds[ap_threads(W) / 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (!FP8 || (int)blockIdx.x < a.row_blocks) append_rows<Tag, D, FP8, NEIGHBOURS, W>(a, lane, wave);
  else append_unit<Tag, D, NEIGHBOURS, W>(a, lane, wave, lds);
}

template <typename Tag, int D, bool FP8, bool NEIGHBOURS, int W>
int launch_append_w(Append a, int64_t rows, int64_t units, hipStream_t s) {
  constexpr int WAVES = ap_threads(W) / 64;
  const int64_t row_blocks = rows ? ((int64_t)a.T * a.parts + WAVES - 1) / WAVES : 0, unit_blocks = (units * W + WAVES - 1) / WAVES;
  if (!launch_fits(row_blocks + unit_blocks, WAVES * 64)) return MLT_ERR_UNSUPPORTED;      // (with it wavefronts, and units, are counted in 32 bits)
  if (row_blocks + unit_blocks == 0) return MLT_OK;
  a.row_blocks = (int)row_blocks;
  hipLaunchKernelGGL((append_kernel<Tag, D, FP8, NEIGHBOURS, W>), dim3((unsigned)(row_blocks + unit_blocks)), dim3(WAVES * 64), 0, s, a);
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

template <typename Tag, int D, bool FP8, bool NEIGHBOURS>
int launch_append(const AppendArgs& g, hipStream_t s) {
  Append a{(int)g.T, (int)g.B, (int)g.Hq, (int)g.H, (int)g.block_size, (int)g.max_blocks, (int)g.num_blocks, (int)(g.rot / 2), (int)g.positions, 0, 1, 0,
           g.Q, g.ldq, g.K, g.ldk, g.V, g.ldv, g.offsets, g.seq_lens, g.block_table, g.cos, g.sin, g.Qo, g.Kc, g.Vc, g.Ks, g.Vs};
  constexpr int RPI = 512 / D;
  const int64_t rows = FP8 ? g.Hq : g.Hq + 2 * g.H;
  // a token's rows over several wavefronts where there are few tokens
  while (a.parts < 16 && g.T * a.parts < 2048 && rows > RPI * a.parts) a.parts *= 2;
  if (!FP8) return launch_append_w<Tag, D, FP8, NEIGHBOURS, 1>(a, rows, 0, s);
  const int64_t by_block = g.T / g.block_size + 2 * g.B;
  a.dense_items = g.T <= by_block;
  const int64_t units = (a.dense_items ? g.T : by_block) * 2 * g.H;
  // As many wavefronts to a unit as hold its new tokens in registers, 16 each (8191 tokens, 8 heads of 128, blocks of 32, 64, 128: 37.2, 37.5, 39.9 us; with four
  // wavefronts 42.2, 37.5, 45.2; with one 43.7, 51.2, 72.8); one for single tokens, whatever the block size (255 tokens, 16 heads: 10.8 us, with four 28.3)
  const int64_t w = a.dense_items ? 1 : g.block_size / 16;
  if (w <= 1) return launch_append_w<Tag, D, true, NEIGHBOURS, 1>(a, rows, units, s);
  if (w <= 2) return launch_append_w<Tag, D, true, NEIGHBOURS, 2>(a, rows, units, s);
  if (w <= 4) return launch_append_w<Tag, D, true, NEIGHBOURS, 4>(a, rows, units, s);
  if (w <= 8) return launch_append_w<Tag, D, true, NEIGHBOURS, 8>(a, rows, units, s);
  return launch_append_w<Tag, D, true, NEIGHBOURS, 16>(a, rows, units, s);
}

template <typename Tag, int D>
int run_append_t(const AppendArgs& a, bool fp8, hipStream_t s) {
  if (fp8) return a.interleaved ? launch_append<Tag, D, true, true>(a, s) : launch_append<Tag, D, true, false>(a, s);
  return a.interleaved ? launch_append<Tag, D, false, true>(a, s) : launch_append<Tag, D, false, false>(a, s);
}

}  // namespace

int run_append(const AppendArgs& a, bool fp8, hipStream_t s) {
  if (a.dtype == MLT_BF16) return a.D == 128 ? run_append_t<bf16_tag, 128>(a, fp8, s) : run_append_t<bf16_tag, 64>(a, fp8, s);
  return a.D == 128 ? run_append_t<f16_tag, 128>(a, fp8, s) : run_append_t<f16_tag, 64>(a, fp8, s);
}

}  // namespace mlt
