// mlt_gemm_fp8 with few rows (next-token decode) or little work: the design of gemm_skinny.hip on e4m3 operands. The cost is reading B once:
// one workgroup of 8 wavefronts per CU, each with its share of the columns (rows of the stored B) in blocks of up to 16; the
// wavefronts split K in pieces of 256 k, 256 bytes a row and two scale blocks. Every wavefront fetches its pieces of A and B
// straight into an LDS ring of its own, several slots ahead, waits for the oldest by count and multiplies: two MFMAs of 128 k for a piece of
// a 16 x 16 tile, each with its scales. Rows are stored permuted (chunk c of row r at position c ^ r), and a wavefront starts some
// pieces into its share and goes round, as there.
//
// The scales come in the same stream: an A slot has 256 bytes more, one direct load of a dword a lane, with the scales of its 16
// rows for the two blocks (lanes 0 .. 31) and those of the columns (lanes 32 .. 35: two blocks of k, two blocks of n; a workgroup's
// group of columns is at most 128 wide and so touches two).
//
// With few columns a CU fetches more of A than of B; K may then be split over 2, 4 or 8 workgroups (PARTS), whose fp32 partial results
// the one that comes last at a counter adds in the order of the parts. More than 64 rows are shared out to rows of workgroups, which read B once
// each: a matrix too small to give every CU a tile of 128 x 128 is better off with 64 x 16 and no barrier in the loop over K.
//
// Measured: 16 x 4096 x 4096 5.0 us, 24 x 14336 x 4096 12.4 us (59 MB, 4.8 TB/s), 65 x 8192 x 1024 7.3 us, 512 x 512 x 1024 5.0 us.
#include "fp8.h"
#include "mlt_internal.h"

namespace mlt {

namespace {

constexpr int S8_NW = 8;              // wavefronts per workgroup = K split
constexpr int S8_NT = S8_NW * 64;
constexpr int S8_KP = 256;            // k values per piece
constexpr int S8_RING = 20 * 1024;    // LDS ring of a wavefront
constexpr int S8_SMEM = S8_NW * S8_RING;

// MT: 16-row tiles of A. AU, BU: load instructions (4 rows each) for a piece of a row tile, of a column block: 4, or fewer where no more rows
// or columns exist
template <int MT, int AU, int BU> struct S8Cfg {
  static constexpr int LU = AU > BU ? AU : BU;
  static constexpr int SLOT = LU * 1024 + 256;
  static constexpr int R = S8_RING / SLOT < 12 ? S8_RING / SLOT : 12;     // slots
  static constexpr int CB = 4 * BU;                                       // columns per block
  static constexpr int MAX_GB = BU < 4 ? 1 : MT <= 2 ? 8 : 4;             // blocks per group, at most
  static_assert(MAX_GB * MT * 1024 <= S8_RING, "a wavefront's partial tiles lie in its own ring");
  static_assert(MAX_GB * CB <= 128, "a group of columns touches at most two scale blocks");
  static_assert(R * (LU + 1) < 63, "loads in flight are counted");
};

struct S8 {
  int M, N, K, rows, share, rest, lda, ldb, nz, nxcd;
  const uint8_t *A, *B;
  const float *Sa, *Sb;
  int64_t ldsa, ldsb;
  uint16_t* C;
  int64_t ldc;
  float* part;
  uint32_t* counter;
};

template <typename Tag, int MT, int AU, int BU, bool PARTS, int GB>
__global__ __launch_bounds__(S8_NT, 2) void gemm_fp8_skinny_kernel(S8 a) {
  typedef S8Cfg<MT, AU, BU> L;
  constexpr int CB = L::CB, R = L::R;
  extern __shared__ __align__(16) char smem[];
  // share of the columns, of the rows, part of K. With several shares of the rows an XCD gets all of them for neighbouring columns of one part (777 x 2048 x 8192: 43 us,
  // 53 with the columns in turn)
  int bid = (int)blockIdx.x, z = 0, part_id = (int)blockIdx.y;
  if (a.nz > 1) {
    const int width = (int)gridDim.x, l = logical_block(bid + part_id * width, width * (int)gridDim.y, a.nxcd);
    part_id = PARTS ? l / width : 0;
    const int at = l - part_id * width;
    bid = at / a.nz;
    z = at - bid * a.nz;
  }
  const int m0 = z * a.rows, M = a.M - m0 < a.rows ? a.M - m0 : a.rows, N = a.N, K = a.K;   // this workgroup's rows
  const uint8_t* const A = a.A + (int64_t)m0 * (uint32_t)a.lda;
  const float* const Sa = a.Sa + m0;
  uint16_t* const C = a.C + (int64_t)m0 * a.ldc;
  const int64_t part_size = (int64_t)a.M * N;
  float* const part = PARTS ? a.part + (int64_t)m0 * N : nullptr;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, q = lane >> 4;
  const int c0 = bid * a.share + (bid < a.rest ? bid : a.rest), c1 = c0 + a.share + (bid < a.rest ? 1 : 0);
  const int nblk = GB == 1 ? 1 : (c1 - c0 + CB - 1) / CB;
  // pieces p0 .. p1 - 1, of them first = p0 + wave, first + 8, ..., from `start` on and then from the first again
  int p0 = 0, p1 = (K + S8_KP - 1) / S8_KP;
  if (PARTS) {
    const int per = (p1 + (int)gridDim.y - 1) / (int)gridDim.y;
    p0 = part_id * per;
    p1 = p0 + per < p1 ? p0 + per : p1;
  }
  const int first = p0 + wave, mine = p1 > first ? (p1 - first + S8_NW - 1) / S8_NW : 0;
  const bool shared_lines = ((reinterpret_cast<uintptr_t>(a.B) | (uintptr_t)(uint32_t)a.ldb) & 63) != 0;
  const int start = first + (shared_lines ? 0 : wave & (mine >= 8 ? 7 : mine >= 4 ? 3 : mine >= 2 ? 1 : 0)) * S8_NW;
  const uint32_t ring = (uint32_t)(uintptr_t)(lptr_t)smem + (uint32_t)wave * S8_RING;
  const int last_kb = (K + F8_KB - 1) / F8_KB - 1;

  // load instruction i of a slot: rows 4 i .. 4 i + 3, lane l the chunk at position l % 16 of row 4 i + l / 16
  uint32_t va[AU], vb[BU];
#pragma unroll
  for (int i = 0; i < AU; ++i)
    va[i] = (uint32_t)(i * 4 + lane / 16) * (uint32_t)a.lda + (uint32_t)((lane % 16) ^ (i * 4 + lane / 16)) * 16u;
#pragma unroll
  for (int i = 0; i < BU; ++i)
    vb[i] = (uint32_t)(i * 4 + lane / 16) * (uint32_t)a.ldb + (uint32_t)((lane % 16) ^ (i * 4 + lane / 16)) * 16u;

  for (int base = 0; base < nblk; base += GB) {
    const int nb = GB == 1 ? 1 : nblk - base < GB ? nblk - base : GB;
    const int S = MT + nb, T = mine * S;                 // slots per piece (row tiles, then column blocks), in all
    const int nblock0 = (c0 + base * CB) / 128, nblock_last = (N - 1) / 128;
    // where this lane's scales lie: rows of A (less 16 * row tile) or a block of columns, and which of a piece's two k blocks
    const int nblock = nblock0 + (lane & 1) < nblock_last ? nblock0 + (lane & 1) : nblock_last;
    const float* sp = lane < 32 ? Sa : a.Sb + nblock;
    const int64_t sld = lane < 32 ? a.ldsa : a.ldsb;
    const int skb = lane < 32 ? lane >> 4 : (lane >> 1) & 1;
    f32x4 acc[GB][MT];
#pragma unroll
    for (int gb = 0; gb < GB; ++gb)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) acc[gb][mt] = f32x4{0.f, 0.f, 0.f, 0.f};

    // the cursor: the next slot of the stream to fetch, f_s of piece f_p, and its place
    int f_t = 0, f_s = 0, f_p = start;
    uint32_t f_slot = ring;
    int issued = 0, need = 0;                            // load instructions issued; up to the end of the slot in hand
    auto fetch = [&]() __attribute__((always_inline)) {
      if (f_t >= T) return;
      const int k0 = f_p * S8_KP;
      const bool tail = k0 + S8_KP > K;
      // rows past the matrix (past this workgroup's columns) and chunks past K: the piece's first chunk for all such
      // lanes, never stored or zeroed later; the instruction stays, and with it the count of loads in flight
      if (f_s < MT) {
        // (the last workgroups' rows may end before a row tile: then all lanes read the first row's chunk)
        const int rows = M - f_s * 16;
        const char* src = reinterpret_cast<const char*>(A + (int64_t)(rows > 0 ? f_s * 16 : 0) * (uint32_t)a.lda + k0);
#pragma unroll
        for (int i = 0; i < AU; ++i) {
          const int row = i * 4 + lane / 16;
          uint32_t off = row < rows ? va[i] : 0u;
          if (tail && k0 + ((lane % 16) ^ row) * 16 >= K) off = 0u;
          load_lds16(src, off, f_slot + i * 1024u);
        }
        const int kb = 2 * f_p + skb < last_kb ? 2 * f_p + skb : last_kb;
        const int row = f_s * 16 + r16 < M ? f_s * 16 + r16 : M - 1;
        load_lds4(sp + kb * sld + (lane < 32 ? row : 0), f_slot + L::LU * 1024u);
        issued += AU + 1;
      } else {
        const int n0 = c0 + (base + f_s - MT) * CB;
        const char* src = reinterpret_cast<const char*>(a.B + (int64_t)n0 * (uint32_t)a.ldb + k0);
        const int rows = c1 - n0;
#pragma unroll
        for (int i = 0; i < BU; ++i) {
          const int row = i * 4 + lane / 16;
          uint32_t off = row < rows ? vb[i] : 0u;
          if (tail && k0 + ((lane % 16) ^ row) * 16 >= K) off = 0u;
          load_lds16_stream(src, off, f_slot + i * 1024u);
        }
        issued += BU;
      }
      ++f_t;
      f_slot = f_slot == ring + (R - 1) * L::SLOT ? ring : f_slot + L::SLOT;
      if (++f_s == S) {
        f_s = 0;
        f_p = f_p + S8_NW < p1 ? f_p + S8_NW : first;
      }
    };
#pragma unroll
    for (int i = 0; i < R; ++i) fetch();

    // the next slot, of n loads: wait until it has landed (what was issued after it may be in flight), read its
    // fragments, refill its place
    uint32_t slot = ring;
    auto take = [&](u32x4 (&f)[4], int n, int loads, auto&& scales) __attribute__((always_inline)) {
      need += loads;
      int later = issued - need;
#ifdef MLT_DEBUG_BARRIERS
      later = 0;                                         // waits for all of them, so that a count that is too lax shows
#endif
      if (L::LU == 4 && later >= 12) __builtin_amdgcn_s_waitcnt(wait_imm(12, 15));
      else if (later >= 10) __builtin_amdgcn_s_waitcnt(wait_imm(10, 15));
      else if (later >= 8) __builtin_amdgcn_s_waitcnt(wait_imm(8, 15));
      else if (later >= 6) __builtin_amdgcn_s_waitcnt(wait_imm(6, 15));
      else if (later >= 4) __builtin_amdgcn_s_waitcnt(wait_imm(4, 15));
      else if (later >= 2) __builtin_amdgcn_s_waitcnt(wait_imm(2, 15));
      else if (later >= 1) __builtin_amdgcn_s_waitcnt(wait_imm(1, 15));
      else __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));
      __builtin_amdgcn_sched_barrier(0);
      const int row = r16 & (4 * n - 1);                 // (fewer than 16 rows: repeated, never stored)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        f[j] = *(const MLT_LDS u32x4*)(uintptr_t)(slot + (uint32_t)row * 256u + (uint32_t)(((j * 4 + q) ^ row) << 4));
      scales(slot + L::LU * 1024u);
      __builtin_amdgcn_s_waitcnt(wait_imm(63, 0));
      __builtin_amdgcn_sched_barrier(0);
      fetch();
      __builtin_amdgcn_sched_barrier(0);
      slot = slot == ring + (R - 1) * L::SLOT ? ring : slot + L::SLOT;
    };
    const u32x4 zero4 = {0u, 0u, 0u, 0u};
    for (int i = 0, piece = start; i < mine; ++i, piece = piece + S8_NW < p1 ? piece + S8_NW : first) {
      const int k0 = piece * S8_KP;
      const bool tail = k0 + S8_KP > K;                  // chunks past K: zeros in both operands
      u32x4 af[MT][4], sb4;                              // sb4: k block 0 with column blocks 0, 1, then k block 1
      f32x4 sa[MT][2];                                   // rows 4 q .. 4 q + 3 of each k block
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        take(af[mt], AU, AU + 1, [&](uint32_t at) __attribute__((always_inline)) {
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) sa[mt][kb] = *(const MLT_LDS f32x4*)(uintptr_t)(at + kb * 64u + q * 16u);
          if (mt == 0) sb4 = *(const MLT_LDS u32x4*)(uintptr_t)(at + 128u);
        });
      if (tail) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (k0 + (j * 4 + q) * 16 >= K) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) af[mt][j] = zero4;
          }
      }
#pragma unroll
      for (int gb = 0; gb < GB; ++gb)
        if (gb < nb) {
          u32x4 bf[4];
          take(bf, BU, BU, [](uint32_t) __attribute__((always_inline)) {});
          if (tail) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (k0 + (j * 4 + q) * 16 >= K) bf[j] = zero4;
          }
          const bool next = (c0 + (base + gb) * CB + r16) / 128 > nblock0;   // this lane's column: in the second column block
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) {
            const float sb = __builtin_bit_cast(float, next ? sb4[2 * kb + 1] : sb4[2 * kb]);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              const f32x4 p = mfma16_e4m3(af[mt][2 * kb], af[mt][2 * kb + 1], bf[2 * kb], bf[2 * kb + 1], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
              for (int r = 0; r < 4; ++r) acc[gb][mt][r] += p[r] * (sa[mt][kb][r] * sb);
            }
          }
        }
    }
    // the partial tiles into the wavefront's own ring (all its loads have landed), then their sums
    float* own = reinterpret_cast<float*>(smem + wave * S8_RING);
#pragma unroll
    for (int gb = 0; gb < GB; ++gb)
      if (gb < nb) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int r = 0; r < 4; ++r) own[(gb * MT + mt) * 256 + (4 * q + r) * 16 + r16] = acc[gb][mt][r];
      }
    __syncthreads();
    for (int e = tid; e < nb * MT * 256; e += S8_NT) {
      const int t = e >> 8, gr = t % MT * 16 + ((e >> 4) & 15), gc = c0 + (base + t / MT) * CB + (e & 15);
      if (gr < M && gc < c1 && (e & 15) < CB) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < S8_NW; ++w) sum += reinterpret_cast<const float*>(smem)[w * (S8_RING / 4) + e];
        if (PARTS) store_shared(part + part_id * part_size + (int64_t)gr * N + gc, sum);
        else C[(int64_t)gr * a.ldc + gc] = Elem<Tag>::from_f32(sum);
      }
    }
    if (base + GB < nblk) __syncthreads();
  }
  if (!PARTS) return;

  // the last part of these columns to get here adds them all (EB elements of a thread at a time, all their parts requested
  // before the first is used: each such round is a trip to memory)
  if (!last_to_arrive(a.counter + bid * a.nz + z, gridDim.y, reinterpret_cast<uint32_t*>(smem))) return;
  const int cols = c1 - c0, parts = (int)gridDim.y;
  constexpr int EB = MT == 1 ? 2 : 4;
  for (int e0 = tid; e0 < M * cols; e0 += EB * S8_NT) {
    float v[8][EB];
    int64_t at[EB];
#pragma unroll
    for (int i = 0; i < EB; ++i) {
      const int e = e0 + i * S8_NT < M * cols ? e0 + i * S8_NT : e0;
      at[i] = (int64_t)(e / cols) * N + c0 + e % cols;
    }
#pragma unroll
    for (int p = 0; p < 8; ++p)
      if (p < parts) {
#pragma unroll
        for (int i = 0; i < EB; ++i) v[p][i] = load_shared(part + p * part_size + at[i]);
      }
#pragma unroll
    for (int p = 1; p < 8; ++p)
      if (p < parts) {
#pragma unroll
        for (int i = 0; i < EB; ++i) v[0][i] += v[p][i];
      }
#pragma unroll
    for (int i = 0; i < EB; ++i)
      if (e0 + i * S8_NT < M * cols) {
        const int gr = (e0 + i * S8_NT) / cols, gc = c0 + (e0 + i * S8_NT) % cols;
        C[(int64_t)gr * a.ldc + gc] = Elem<Tag>::from_f32(v[0][i]);
      }
  }
}

template <typename Tag, int MT, int AU, int BU, bool PARTS, int GB>
int launch_s8_blocks(const GemmFp8Args& g, int rows, int parts, float* part, unsigned nwg, hipStream_t s) {
  auto kern = gemm_fp8_skinny_kernel<Tag, MT, AU, BU, PARTS, GB>;
  static thread_local int configured_dev = -1;            // opt in to > 64 KB LDS once per device
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return MLT_ERR_DEVICE;
  if (configured_dev != dev) {
    if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, S8_SMEM) != hipSuccess) {
      (void)hipGetLastError();
      return MLT_ERR_LAUNCH;
    }
    configured_dev = dev;
  }
  S8 a{(int)g.M, (int)g.N, (int)g.K, rows, (int)(g.N / nwg), (int)(g.N % nwg), (int)g.lda, (int)g.ldb, (int)((g.M + rows - 1) / rows), device_xcds(), g.A, g.B, g.Sa, g.Sb, g.ldsa, g.ldsb, g.C, g.ldc, part,
       PARTS ? scratch_counters(part) : nullptr};
  hipLaunchKernelGGL(kern, dim3(nwg * (unsigned)a.nz, (unsigned)parts), dim3(S8_NT), S8_SMEM, s, a);
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

template <typename Tag, int MT, int AU, int BU, bool PARTS>
int launch_s8(const GemmFp8Args& g, int rows, int parts, float* part, int64_t ncu, hipStream_t s) {
  constexpr int MAX_GB = S8Cfg<MT, AU, BU>::MAX_GB;
  const int64_t per = parts * ((g.M + rows - 1) / rows), want = ncu / per > 0 ? ncu / per : 1;
  const unsigned nwg = (unsigned)(g.N < want ? g.N : want);   // one workgroup per CU, every one with columns
  const int64_t blocks = ((g.N + nwg - 1) / nwg + 4 * BU - 1) / (4 * BU);
  if (blocks == 1) return launch_s8_blocks<Tag, MT, AU, BU, PARTS, 1>(g, rows, parts, part, nwg, s);
  if (blocks == 2 && MAX_GB == 8) return launch_s8_blocks<Tag, MT, AU, BU, PARTS, MAX_GB == 8 ? 2 : MAX_GB>(g, rows, parts, part, nwg, s);
  return launch_s8_blocks<Tag, MT, AU, BU, PARTS, MAX_GB>(g, rows, parts, part, nwg, s);
}

template <typename Tag, int MT, int AU>
int run_s8_cols(const GemmFp8Args& g, int rows, int parts, float* part, int64_t ncu, hipStream_t s) {
  if (parts > 1) return launch_s8<Tag, MT, AU, 4, true>(g, rows, parts, part, ncu, s);
  switch (gemm_skinny_cols(g.N, parts, ncu / ((g.M + rows - 1) / rows))) {
    case 4: return launch_s8<Tag, MT, AU, 1, false>(g, rows, 1, nullptr, ncu, s);
    case 8: return launch_s8<Tag, MT, AU, 2, false>(g, rows, 1, nullptr, ncu, s);
  }
  return launch_s8<Tag, MT, AU, 4, false>(g, rows, 1, nullptr, ncu, s);
}

template <typename Tag>
int run_s8_t(const GemmFp8Args& g, int parts, float* part, int64_t ncu, hipStream_t s) {
  const int rows = gemm_fp8_skinny_rows(g.M);
  if (rows <= 4) return run_s8_cols<Tag, 1, 1>(g, rows, parts, part, ncu, s);
  switch ((rows + 15) / 16) {
    case 1: return run_s8_cols<Tag, 1, 4>(g, rows, parts, part, ncu, s);
    case 2: return run_s8_cols<Tag, 2, 4>(g, rows, parts, part, ncu, s);
    case 3: return run_s8_cols<Tag, 3, 4>(g, rows, parts, part, ncu, s);
    case 4: return run_s8_cols<Tag, 4, 4>(g, rows, parts, part, ncu, s);
  }
  return MLT_ERR_UNSUPPORTED;
}

}  // namespace

int run_gemm_fp8_skinny(const GemmFp8Args& g, int parts, float* part, hipStream_t s) {
  DeviceInfo di;
  const int64_t ncu = device_info(di) && di.ncu > 0 ? di.ncu : 256;
  return g.dtype == MLT_BF16 ? run_s8_t<bf16_tag>(g, parts, part, ncu, s) : run_s8_t<f16_tag>(g, parts, part, ncu, s);
}

}  // namespace mlt
