// C = A * B^T on e4m3 operands with a scale for each block of 128 of K (mlt_gemm_fp8):
//   C[m][n] = sum over blocks kb of Sa[kb][m] * Sb[kb][n / 128] * sum over k in kb of A[m][k] * B[n][k]
// One MFMA (16x16x128) multiplies a block's 128 k of a 16 x 16 tile; its fp32 result, started from zero, goes into the fp32
// accumulator with the product of the two scales. That is four fused multiply-adds behind each MFMA of 32 clocks, which take 16 clocks of
// the vector unit beside it: they are issued two MFMAs late, while later ones run.
//
// The schedule is that of gemm_pp.hip, whose K step of 64 16-bit values has the bytes of a K step of 128 here: workgroup tile 256 x 256
// (or 128 x 128, two workgroups per CU), 8 wavefronts as 2 x 4, the two of a SIMD half a step apart, one refilling its
// fragments from LDS while the other multiplies; direct-to-LDS loads into a ring of five operand tiles A_0 B_0 A_1 B_1 A_2 ...,
// group 1 fetching A and group 0 B; 16-byte chunk c of tile row r at position c ^ ((r >> 1) & 7).
// The ring fills the LDS, so the scales of A go through registers: a lane loads one row's scale (of each 64 of its wavefront's rows) for
// the next step, and swaps between lane groups spread a row's scale over the four groups that hold its results (rows of A are the
// columns of the MFMA, so a lane has one row a tile). Those loads sit in front of the step's direct ones, behind a wait for
// all earlier ones: A of the next step has to have landed by the end of that phase anyway, and B has.
//
// The 128-column tiles (gemm_fp8_kp_kernel) follow gemm_kp.hip: 256 to 128 rows x 128 columns, the two groups on alternate K steps, the scales in the LDS stage of their
// step; K may be split in two parts, joined by the workgroup that comes last, or in up to 8, added by gemm_splitk_reduce_kernel. Which kernel runs is decided by estimated time (fp8_estimate).
//
// Measured: 8192 x 8192 x 8192 423 to 450 us by the board, 2440 to 2600 TFLOP/s (485 in a row of its own, at the power cap); 777 x 4096 x 14336 59 to 65 us by 224 x 128 tiles
// and two parts, 1400 to 1540 TFLOP/s (its direct loads with barriers alone take 49 us, its MFMAs with barriers alone 48). A K step of a 256 x 256 tile, 1.98 us on random bits (1.65 on quantised N(0, 1)):
// the MFMAs and barriers alone take 1.36, all but the direct loads 1.55, with sums by the MFMA itself (one scale for all of K) 1.76. It is 3250 clocks at the 1.8 GHz that the
// board's power leaves: 2048 of the matrix units and as many of the LDS (192 KB of fragments read, 64 KB written, 128 bytes a clock).
#include <stdio.h>

#include "fp8.h"
#include "mlt_internal.h"

namespace mlt {

namespace {

constexpr int G8_NT = 512;
constexpr int G8_NSLOT = 5;
constexpr int G8_GROUP_M = 4;              // as in gemm_pp.hip
template <int BT> struct G8Tile {
  static constexpr int SLOT = BT * F8_KB;
  static constexpr int SMEM = G8_NSLOT * SLOT;
  static constexpr int NL = SLOT / 1024 / 4;             // 1 KB blocks (8 rows) per wavefront and tile
};

// Lane groups (16 lanes each) 0 1 2 3 of x -> out[g]: group g in all four
__device__ __forceinline__ void spread_groups(float x, float (&out)[4]) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto h = __builtin_amdgcn_permlane32_swap(u, u, false, false);       // 0 1 0 1 | 2 3 2 3
  const auto a = __builtin_amdgcn_permlane16_swap(h[0], h[0], false, false); // 0 0 0 0 | 1 1 1 1
  const auto b = __builtin_amdgcn_permlane16_swap(h[1], h[1], false, false);
  out[0] = __builtin_bit_cast(float, (unsigned)a[0]);
  out[1] = __builtin_bit_cast(float, (unsigned)a[1]);
  out[2] = __builtin_bit_cast(float, (unsigned)b[0]);
  out[3] = __builtin_bit_cast(float, (unsigned)b[1]);
}

// N blocks (8 tile rows of 128 bytes each) from `first` on, of a tile whose row 0 lies at gp (at this K step) and whose last row inside the matrix is `last`, into LDS:
// lane l fetches the 16 bytes that belong at dst + 1024 i + 16 l, chunk (l & 7) ^ ((r >> 1) & 7) of row r. Rows past the matrix read its last rows again, chunks past
// k_left (TAIL) the row's first; what lands there is never stored, or zeroed in the fragments. The lane's offset has two forms, for even and odd blocks; the rows go
// into the scalar base: a load costs no vector instruction, which would stand in the memory phase's way (computed per load: 256 x 128 tiles 29 %
// more time), and no register through the loop.
// between(i) is called behind load i: the LDS reads of a memory phase go there, on a path of their own.
template <int N, bool TAIL, typename Between>
__device__ __forceinline__ void load_blocks(const char* gp, uint32_t ld, int last, int first, uint32_t dst, int lane, bool stream, int k_left, Between&& between) {
  int ln = lane;
  asm volatile("" : "+v"(ln));
  uint32_t c0 = (uint32_t)((ln & 7) ^ (((ln >> 4) | (first << 2)) & 7)) * 16u, c1 = c0 ^ 64u;
  if (TAIL) {
    c0 = (int)c0 < k_left ? c0 : 0u;
    c1 = (int)c1 < k_left ? c1 : 0u;
  }
  const uint32_t row = (uint32_t)(ln >> 3) * ld, v0 = row + c0, v1 = row + c1;
  if ((first + N) * 8 - 1 <= last) {
    const char* p = gp + (int64_t)(first * 8) * ld;
    if (stream) {
#pragma unroll
      for (int i = 0; i < N; ++i, p += ld * 8) {
        load_lds16_stream(p, i & 1 ? v1 : v0, dst + i * 1024);
        between(i);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i, p += ld * 8) {
        load_lds16(p, i & 1 ? v1 : v0, dst + i * 1024);
        between(i);
      }
    }
  } else {
    const uint32_t edge = (uint32_t)((ln >> 3) < (last & 7) ? ln >> 3 : last & 7) * ld;
    const int lb = last >> 3;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int b = first + i < lb ? first + i : lb;
      load_lds16(gp + (int64_t)(b * 8) * ld, (b == lb ? edge : row) + (i & 1 ? c1 : c0), dst + i * 1024);
      between(i);
    }
  }
}

// One K step of a wavefront's TA x TB tiles: the products of a scale block, and two MFMAs behind each its sum. now: the step's scales, row
// 64 i + lane in now[i].
// (One MFMA behind, a sum waits for its operand: 42 clocks an MFMA instead of 35, of which 32 are the MFMA's own. The empty asm
// statements keep each MFMA and each sum where it is written: behind the last MFMA all parts would be alive.)
template <int TA, int TB>
__device__ __forceinline__ void mul_step(const u32x4 (&af)[2][TA], const u32x4 (&bf)[2][TB], const float (&now)[(TA + 3) / 4], f32x4 (&acc)[TA][TB]) {
  f32x4 late[2];
  float s[4], late_s[2] = {0.f, 0.f};
#pragma unroll
  for (int e = 0; e < TA * TB + 2; ++e) {
    f32x4 part;
    if (e < TA * TB) {
      part = mfma16_e4m3(bf[0][e % TB], bf[1][e % TB], af[0][e / TB], af[1][e / TB], f32x4{0.f, 0.f, 0.f, 0.f});
      asm volatile("" : "+v"(part));
      __builtin_amdgcn_sched_barrier(0);
      if (e % (4 * TB) == 0) spread_groups(now[e / (4 * TB)], s);
    }
    if (e > 1) {
      f32x4& to = acc[(e - 2) / TB][(e - 2) % TB];
#pragma unroll
      for (int r = 0; r < 4; ++r) to[r] += late[e & 1][r] * late_s[e & 1];
      asm volatile("" : "+v"(to));
    }
    late[e & 1] = part;
    late_s[e & 1] = s[e / TB % 4];
    __builtin_amdgcn_sched_barrier(0);
  }
}

}  // namespace

// TAIL: K is no multiple of 128
template <typename Tag, int BT, bool TAIL>
__global__ __launch_bounds__(G8_NT, BT == 128 ? 4 : 1) void gemm_fp8_kernel(int M, int N, int K, const uint8_t* __restrict__ A, int64_t lda, const float* __restrict__ Sa,
                                                                            int64_t ldsa, const uint8_t* __restrict__ B, int64_t ldb, const float* __restrict__ Sb,
                                                                            int64_t ldsb, uint16_t* __restrict__ C, int64_t ldc, int nbm, int nbn, int nxcd) {
  typedef G8Tile<BT> T;
  constexpr int SLOT = T::SLOT, NL = T::NL, WTM = BT / 2, WTN = BT / 4, TA = WTM / 16, TB = WTN / 16;
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 2, wn = wave & 3, grp = wm;
  int tile_m, tile_n;
  tile_of_block<G8_GROUP_M>(blockIdx.x, nbm, nbn, nxcd, tile_m, tile_n);
  const int m0 = tile_m * BT, n0 = tile_n * BT;
  const int KT = (K + F8_KB - 1) / F8_KB;
  const int k_tail = K - (KT - 1) * F8_KB;               // TAIL: k values in the last step

  // ---- global -> LDS: the wavefronts of group 1 fill the A tiles, those of group 0 the B tiles, NL blocks of 8 rows each
  const char* ld_base = reinterpret_cast<const char*>(grp ? A + (int64_t)m0 * lda : B + (int64_t)n0 * ldb);
  const uint32_t ld_row = (uint32_t)(grp ? lda : ldb);
  const int ld_last = (grp ? M - m0 : N - n0) - 1;       // last row inside the matrix
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lptr_t)smem;
  const bool stream = grp == 1 ? nbn == 1 : nbm == 1;    // (read once: streaming form)
  auto issue_loads = [&](int t, int slot, auto&& between) __attribute__((always_inline)) {
    load_blocks<NL, TAIL>(ld_base + (int64_t)t * F8_KB, ld_row, ld_last, (wave & 3) * NL, lds0 + slot * SLOT + (wave & 3) * (NL * 1024), lane, stream, K - t * F8_KB, between);
  };
  auto nothing = [](int) __attribute__((always_inline)) {};

  // ---- scales: of row 64 i + lane of this wavefront's rows (with 64 rows: i = 0), and of the block of its columns
  constexpr int NS = WTM / 64;
  uint32_t srow[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const int r = m0 + wm * WTM + 64 * i + lane;
    srow[i] = (uint32_t)(r < M ? r : M - 1);
  }
  const int ncol = n0 + wn * WTN < N ? n0 + wn * WTN : N - 1;
  const int scol = ncol / F8_KB;
  float sa[NS], sb;
  auto load_scales = [&](int t) {
#pragma unroll
    for (int i = 0; i < NS; ++i) sa[i] = (Sa + (int64_t)t * ldsa)[srow[i]];
    sb = (Sb + (int64_t)t * ldsb)[scol];
  };

  // ---- fragments: chunks h and 4 + h of a tile's rows
  const int lq = lane & 15, h = lane >> 4;
  const int swz = (lq >> 1) & 7;
  int a_off[2], b_off[2];
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    a_off[kk] = (wm * WTM + lq) * F8_KB + (((4 * kk + h) ^ swz) * 16);
    b_off[kk] = (wn * WTN + lq) * F8_KB + (((4 * kk + h) ^ swz) * 16);
  }
  f32x4 acc[TA][TB];
#pragma unroll
  for (int i = 0; i < TA; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 af[2][TA], bf[2][TB];
  // fragment f of 2 * (TA + TB): B's first, then A's in the order in which they are multiplied
  auto read_frag = [&](const char* ta, const char* tb, int f) __attribute__((always_inline)) {
    const int kk = f & 1, i = f >> 1;
    if (i < TB) bf[kk][i] = lds_read8<u32x4>(tb, b_off[kk] + i * 16 * F8_KB);
    else af[kk][i - TB] = lds_read8<u32x4>(ta, a_off[kk] + (i - TB) * 16 * F8_KB);
  };
  auto zero_tail = [&]() {                               // both operands: one alone would leave 0 * NaN
    const u32x4 zero4 = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
      if ((4 * kk + h) * 16 >= k_tail) {
#pragma unroll
        for (int i = 0; i < TA; ++i) af[kk][i] = zero4;
#pragma unroll
        for (int j = 0; j < TB; ++j) bf[kk][j] = zero4;
      }
  };

  // Phases and slots as in gemm_pp.hip. Phase p ends at workgroup barrier p. Group 0 reads A_k and B_k in phase 2k and multiplies in
  // phase 2k+1, group 1 one phase later. Operand tile number t (A_k: 2k, B_k: 2k+1) lives in slot t % 5 and is last read in phase 2k+1.
  //   group 1, memory phase of step k (2k+1): waits for A_{k+1}, issued one step earlier, then issues A_{k+2} into the slot that
  //     B_{k-1} left in phase 2k-1;
  //   group 0, memory phase of step k (2k): issues B_{k+1} into the slot that A_{k-1} left in phase 2k-1, and waits for it at
  //     the end of its compute phase.
  load_scales(0);
  issue_loads(0, grp ? 0 : 1, nothing);
  if (KT > 1) { issue_loads(1, grp ? 2 : 3, nothing); __builtin_amdgcn_s_waitcnt(wait_imm(NL, 0)); }
  else __builtin_amdgcn_s_waitcnt(wait_imm(0, 0));
  MLT_BARRIER();
  if (grp == 1) MLT_BARRIER();

  int slot_a = 0;                                         // slot of A_k; B_k is in the next one
#pragma clang loop unroll(disable)                         // (nor a first iteration peeled off: its copy of the fragments does not fit)
  for (int k = 0; k < KT; ++k) {
    const int slot_b = slot_a + 1 == G8_NSLOT ? 0 : slot_a + 1;
    // ---- memory phase
    __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));          // group 1: A_{k+1}; both: the scales of step k
    __builtin_amdgcn_sched_barrier(0);
    float now[NS];                                        // this step's scales, row by lane
#pragma unroll
    for (int i = 0; i < NS; ++i) now[i] = sa[i] * sb;
    if (k + 1 < KT) load_scales(k + 1);
    __builtin_amdgcn_sched_barrier(0);
    const char *ta = smem + slot_a * SLOT, *tb = smem + slot_b * SLOT;
    constexpr int NF = 2 * (TA + TB), PER = NF / NL;
    static_assert(NF % NL == 0, "fragments behind each load");
    const int next = grp == 1 ? (k + 2 < KT ? k + 2 : 0) : (k >= 1 && k + 1 < KT ? k + 1 : 0);
    if (next) {
      const int to = grp == 1 ? slot_a + 4 : slot_a + 3;
      issue_loads(next, to >= G8_NSLOT ? to - G8_NSLOT : to, [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int f = 0; f < PER; ++f) read_frag(ta, tb, i * PER + f);
      });
    } else {
#pragma unroll
      for (int f = 0; f < NF; ++f) read_frag(ta, tb, f);
    }
    __builtin_amdgcn_s_waitcnt(wait_imm(63, 0));
    if (TAIL && k == KT - 1) zero_tail();
    MLT_BARRIER();
    __builtin_amdgcn_sched_barrier(0);
    // ---- compute phase
    mul_step<TA, TB>(af, bf, now, acc);
    if (grp == 0) __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));
    MLT_BARRIER();
    __builtin_amdgcn_sched_barrier(0);
    slot_a = slot_a + 2 >= G8_NSLOT ? slot_a + 2 - G8_NSLOT : slot_a + 2;
  }
  if (grp == 0) MLT_BARRIER();

  // ---- epilogue: through LDS (every wavefront is past its last fragment read), out along the rows
  constexpr int RP = 64;
  typedef RowStore<Tag, RP, WTN, 4> Rows;
  static_assert(8 * Rows::BYTES <= T::SMEM, "one parking area per wavefront");
  float* park = reinterpret_cast<float*>(smem + wave * Rows::BYTES);
#pragma unroll
  for (int p = 0; p < WTM / RP; ++p)
    Rows::run([&](float* lds) {
      // register r of a tile is column 4 h + r of row lq
#pragma unroll
      for (int i = 0; i < RP / 16; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j)
          *reinterpret_cast<f32x4_mem*>(lds + (i * 16 + lq) * Rows::STRIDE + j * 16 + 4 * h) = acc[p * (RP / 16) + i][j];
    }, park, lane, m0 + wm * WTM + p * RP, n0 + wn * WTN, M, N, C, ldc, 0, nullptr);
}

namespace {

// ---- the tiles of gemm_kp.hip: BM x 128, two groups of 4 wavefronts (2 x 2, BM/2 x 64 each) on alternate K steps, whose accumulators
// are added through LDS at the end. Step s is read in phase s and multiplied in phase s + 1 by group s % 2. For grids that do not fill the chip with
// 256 x 256 tiles: as many bytes of fragments per multiplication as there, and K may be split over workgroups (part_steps > 0), which
// leave fp32 partial results.
// A ring of R stages of one K step each (A tile, B tile, their scales); step s + R - 1 is fetched in phase s, by the group whose memory phase that is, into the
// stage that the other one has read in phase s - 1. With R = 3 that is the group that will read it, which waits for it at the end of its compute phase, one phase
// after the loads; with R = 4 it has two phases, and the wait stands at the end of the memory phase, behind the next loads. A phase of the
// shorter tiles is less than the way from memory: R = 4 for them, what fits of the taller ones.
template <int BM> struct K8Tile {
  static constexpr int A_B = BM * F8_KB, B_B = 128 * F8_KB, S_B = 1024, STAGE = A_B + B_B + S_B;
  static constexpr int R = 4 * STAGE <= 160 * 1024 ? 4 : 3;
  static constexpr int NLA = A_B / 1024 / 4, NLB = B_B / 1024 / 4;       // 1 KB loads (8 rows) per wavefront of the group and step
  static constexpr int NL = NLA + NLB + 1;                               // and one of scales
  static constexpr int S = 128 + 4;                                      // floats per row of a group's image of the result
  static constexpr int RPP = BM / 2;                                     // rows per pass of the epilogue
  static constexpr int EP = (RPP * 16 + G8_NT - 1) / G8_NT;              // pieces of 8 columns per thread and pass
  static constexpr int PART = 2 * EP * 8 * G8_NT;                        // floats of a part of a tile
  static constexpr int IMG_B = 2 * RPP * S * 4;
  static constexpr int SMEM = R * STAGE > IMG_B ? R * STAGE : IMG_B;
};

}  // namespace

template <typename Tag, int BM, bool TAIL>
__global__ __launch_bounds__(G8_NT, 2) void gemm_fp8_kp_kernel(int M, int N, int K_, const uint8_t* __restrict__ A, int64_t lda, const float* __restrict__ Sa, int64_t ldsa,
                                                               const uint8_t* __restrict__ B, int64_t ldb, const float* __restrict__ Sb, int64_t ldsb, uint16_t* __restrict__ C,
                                                               int64_t ldc, int nbm, int nbn, int nxcd, int part_steps, int joined, float* part_out) {
  typedef K8Tile<BM> T;
  constexpr int R = T::R, NL = T::NL, NLA = T::NLA, NLB = T::NLB, WTM = BM / 2, WTN = 64, TA = WTM / 16, TB = WTN / 16;
  extern __shared__ __align__(16) char smem[];
  int K = K_, kb0 = 0;
  const int tiles = nbm * nbn;
  int logical, part = 0;
  if (part_steps > 0) {                                  // an XCD takes the tiles of one part (one row of tiles: the same tiles of all parts)
    if (nbm > 1) {
      logical = logical_block(blockIdx.x, gridDim.x, nxcd);
      part = logical / tiles;
      logical -= part * tiles;
    } else {
      part = blockIdx.x / tiles;
      logical = logical_block(blockIdx.x - part * tiles, tiles, nxcd);
    }
    kb0 = part * part_steps;
    K = K_ - kb0 * F8_KB < part_steps * F8_KB ? K_ - kb0 * F8_KB : part_steps * F8_KB;   // > 0: the host launches no empty part
  } else {
    logical = logical_block(blockIdx.x, tiles, nxcd);
  }
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = wave >> 2, w = wave & 3, wm = w >> 1, wn = w & 1;
  const int tile = logical;
  int tile_m, tile_n;
  tile_of_logical<G8_GROUP_M>(logical, nbm, nbn, tile_m, tile_n);
  const int m0 = tile_m * BM, n0 = tile_n * 128;
  const int KT = (K + F8_KB - 1) / F8_KB;
  const int k_tail = K - (KT - 1) * F8_KB;

  // ---- global -> LDS: wavefront w of a group fills blocks w * NLA .. of A and w * NLB .. of B of a step, and 64 scales: those of the rows 64 w .. of the
  // tile (past its end: never read); the columns' scale comes by a scalar load
  const char* const a_base = reinterpret_cast<const char*>(A + (int64_t)m0 * lda) + (int64_t)kb0 * F8_KB;
  const char* const b_base = reinterpret_cast<const char*>(B + (int64_t)n0 * ldb) + (int64_t)kb0 * F8_KB;
  const int a_last = M - 1 - m0, b_last = N - 1 - n0;
  const bool stream_a = nbn == 1, stream_b = nbm == 1;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lptr_t)smem;
  const uint32_t srow = (uint32_t)(64 * w + lane <= a_last ? 64 * w + lane : a_last) * 4u;   // inside the tile: from row 0 on it would pass 32 bits
  auto issue = [&](int s, int stage, auto&& between) __attribute__((always_inline)) {
    const uint32_t at = lds0 + stage * T::STAGE;
    load_lds4(Sa + (int64_t)(kb0 + s) * ldsa + m0, srow, at + T::A_B + T::B_B + w * 256);
    load_blocks<NLA, TAIL>(a_base + (int64_t)s * F8_KB, (uint32_t)lda, a_last, w * NLA, at + w * (NLA * 1024), lane, stream_a, K - s * F8_KB, between);
    load_blocks<NLB, TAIL>(b_base + (int64_t)s * F8_KB, (uint32_t)ldb, b_last, w * NLB, at + T::A_B + w * (NLB * 1024), lane, stream_b, K - s * F8_KB,
                           [&](int i) __attribute__((always_inline)) { between(NLA + i); });
  };
  auto nothing = [](int) __attribute__((always_inline)) {};
  constexpr int NS = (WTM + 63) / 64;
  const float* sb_at = Sb + tile_n;                      // (128 columns: one block)

  const int lq = lane & 15, h = lane >> 4, swz = (lq >> 1) & 7;
  int a_off[2], b_off[2];
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    a_off[kk] = (wm * WTM + lq) * F8_KB + (((4 * kk + h) ^ swz) * 16);
    b_off[kk] = T::A_B + (wn * WTN + lq) * F8_KB + (((4 * kk + h) ^ swz) * 16);
  }
  f32x4 acc[TA][TB];
#pragma unroll
  for (int i = 0; i < TA; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 af[2][TA], bf[2][TB];

  // the steps before R - 1, as if fetched in the phases before 0
  constexpr bool OWN = R % 2 == 1;                        // a group fetches the steps that it reads
#pragma unroll
  for (int j = 0; j < R - 1; ++j)
    if (((j - (R - 1)) & 1) == grp && j < KT) issue(j, j, nothing);
  // step 0 has to have landed at the first barrier: of its group's loads only those of step 2 may be in flight
  if (!OWN && KT > 2 && grp == 1) __builtin_amdgcn_s_waitcnt(wait_imm(NL, 15));
  else if (grp == (OWN ? 0 : 1)) __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));
  MLT_BARRIER();
  if (grp == 1) {
    if (OWN) __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));
    MLT_BARRIER();
  }
  int stage = grp;
  int ld_stage = (grp + R - 1) % R;                       // of step s + R - 1
#pragma clang loop unroll(disable)
  for (int s = grp; s < KT; s += 2) {
    // ---- memory phase s
    const char* st = smem + stage * T::STAGE;
    const float sb = sb_at[(int64_t)(kb0 + s) * ldsb];
    float now[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) now[i] = reinterpret_cast<const f32_mem*>(st + T::A_B + T::B_B)[wm * WTM + 64 * i + lane];
    constexpr int NF = 2 * (TA + TB);
    auto read_frag = [&](int f) __attribute__((always_inline)) {
      const int kk = f & 1, i = f >> 1;
      if (i < TB) bf[kk][i] = lds_read8<u32x4>(st, b_off[kk] + i * 16 * F8_KB);
      else af[kk][i - TB] = lds_read8<u32x4>(st, a_off[kk] + (i - TB) * 16 * F8_KB);
    };
    if (s + R - 1 < KT) {
      issue(s + R - 1, ld_stage, [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int f = i * NF / (NL - 1); f < (i + 1) * NF / (NL - 1); ++f) read_frag(f);
      });
      if (!OWN) __builtin_amdgcn_s_waitcnt(wait_imm(NL, 15));   // step s + 1, fetched two phases ago
    } else {
#pragma unroll
      for (int f = 0; f < NF; ++f) read_frag(f);
      if (!OWN) __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));
    }
    __builtin_amdgcn_s_waitcnt(wait_imm(63, 0));
#pragma unroll
    for (int i = 0; i < NS; ++i) now[i] *= sb;
    if (TAIL && s == KT - 1) {
      const u32x4 zero4 = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
        if ((4 * kk + h) * 16 >= k_tail) {
#pragma unroll
          for (int i = 0; i < TA; ++i) af[kk][i] = zero4;
#pragma unroll
          for (int j = 0; j < TB; ++j) bf[kk][j] = zero4;
        }
    }
    MLT_BARRIER();
    __builtin_amdgcn_sched_barrier(0);
    // ---- compute phase s + 1 (the memory phase goes first at the issue: with 128 rows ±0, 777 x 4096 x 14336 66.6 -> 64.4 us, 2048 x 4096 x 4096 41.1 -> 39.9)
    if (BM > 128) __builtin_amdgcn_s_setprio(0);
    mul_step<TA, TB>(af, bf, now, acc);
    if (BM > 128) __builtin_amdgcn_s_setprio(1);
    if (OWN) __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));
    MLT_BARRIER();
    __builtin_amdgcn_sched_barrier(0);
    stage = stage + 2 >= R ? stage + 2 - R : stage + 2;
    ld_stage = ld_stage + 2 >= R ? ld_stage + 2 - R : ld_stage + 2;
  }
  if (BM > 128) __builtin_amdgcn_s_setprio(0);
  if ((KT & 1) == grp) MLT_BARRIER();                     // KT + 1 phases for both groups

  // ---- epilogue: RPP rows at a time both groups park their accumulators in images of their own; all threads add the two, 8 columns a piece
  float* const img = reinterpret_cast<float*>(smem);
  constexpr int S = T::S, RPP = T::RPP, EP = T::EP;
  const bool in_rows = part_steps > 0 && !joined;        // a part's sums as rows, for another kernel to add up
  f32x4 sum[BM / RPP][EP][2];
#pragma unroll
  for (int p = 0; p < BM / RPP; ++p) {
    if (p > 0) __syncthreads();
    if (wm == p) {
      float* mine = img + (grp * RPP + lq) * S + wn * WTN + 4 * h;
#pragma unroll
      for (int i = 0; i < TA; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) *reinterpret_cast<f32x4_mem*>(mine + i * 16 * S + j * 16) = acc[i][j];
    }
    __syncthreads();
    if (in_rows) {
      for (int e = tid; e < RPP * 32; e += G8_NT) {
        const int r = e / 32, c = e % 32 * 4, row = m0 + p * RPP + r;
        f32x4 v = *reinterpret_cast<const f32x4_mem*>(img + r * S + c);
        add4(v, *reinterpret_cast<const f32x4_mem*>(img + (RPP + r) * S + c));
        if (row < M && n0 + c < N) store_row4(v, part_out + ((int64_t)part * M + row) * N + n0 + c, N - n0 - c, false);
      }
      continue;
    }
#pragma unroll
    for (int i = 0; i < EP; ++i) {
      const int e = i * G8_NT + tid < RPP * 16 ? i * G8_NT + tid : 0;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float* src = img + e / 16 * S + e % 16 * 8 + 4 * k;
        sum[p][i][k] = *reinterpret_cast<const f32x4_mem*>(src);
        add4(sum[p][i][k], *reinterpret_cast<const f32x4_mem*>(src + RPP * S));
      }
    }
  }
  if (in_rows) return;
  if (joined) {
    // two parts: both leave their sums, a thread's next to those of its neighbours, and the one of a tile that comes last adds the other's (a sum of two has no order)
    auto place = [&](int q) __attribute__((always_inline)) { return part_out + (int64_t)(q * tiles + tile) * T::PART + tid; };
    float* mine = place(part);
#pragma unroll
    for (int p = 0; p < BM / RPP; ++p)
#pragma unroll
      for (int i = 0; i < EP; ++i)
#pragma unroll
        for (int c = 0; c < 8; ++c) store_shared(mine + ((p * EP + i) * 8 + c) * G8_NT, sum[p][i][c / 4][c % 4]);
    if (!last_to_arrive(reinterpret_cast<uint32_t*>(part_out) - kScratchCounters + tile, 2u, reinterpret_cast<uint32_t*>(smem))) return;
    const float* other = place(1 - part);
    float v[BM / RPP][EP][8];
#pragma unroll
    for (int p = 0; p < BM / RPP; ++p)
#pragma unroll
      for (int i = 0; i < EP; ++i)
#pragma unroll
        for (int c = 0; c < 8; ++c) v[p][i][c] = load_shared(other + ((p * EP + i) * 8 + c) * G8_NT);
#pragma unroll
    for (int p = 0; p < BM / RPP; ++p)
#pragma unroll
      for (int i = 0; i < EP; ++i)
#pragma unroll
        for (int c = 0; c < 8; ++c) sum[p][i][c / 4][c % 4] += v[p][i][c];
  }
#pragma unroll
  for (int p = 0; p < BM / RPP; ++p)
#pragma unroll
    for (int i = 0; i < EP; ++i) {
      const int e = i * G8_NT + tid, r = m0 + p * RPP + e / 16, c = n0 + e % 16 * 8;
      if (e < RPP * 16 && r < M && c < N) store_row8<Tag, false>(sum[p][i][0], sum[p][i][1], C + (int64_t)r * ldc + c, N - c, 0, nullptr);
    }
}

namespace {

template <typename Tag, int BT, bool TAIL>
int launch_fp8(const GemmFp8Args& a, hipStream_t s) {
  constexpr int SMEM = G8Tile<BT>::SMEM;
  auto kern = gemm_fp8_kernel<Tag, BT, TAIL>;
  static thread_local int configured_dev = -1;          // opt in to > 64 KB LDS once per device
  int dev = 0;
  const int64_t nbm = (a.M + BT - 1) / BT, nbn = (a.N + BT - 1) / BT;
  if (hipGetDevice(&dev) != hipSuccess) return MLT_ERR_DEVICE;
  if (configured_dev != dev) {
    if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, SMEM) != hipSuccess) {
      (void)hipGetLastError();
      return MLT_ERR_LAUNCH;
    }
    configured_dev = dev;
  }
  hipLaunchKernelGGL(kern, dim3((unsigned)(nbm * nbn)), dim3(G8_NT), SMEM, s, (int)a.M, (int)a.N, (int)a.K, a.A, a.lda, a.Sa, a.ldsa, a.B, a.ldb, a.Sb, a.ldsb, a.C,
                     a.ldc, (int)nbm, (int)nbn, device_xcds());
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

template <typename Tag, int BT>
int run_fp8_tile(const GemmFp8Args& a, hipStream_t s) {
  return a.K % F8_KB ? launch_fp8<Tag, BT, true>(a, s) : launch_fp8<Tag, BT, false>(a, s);
}

template <typename Tag, int BM, bool TAIL>
int launch_fp8_kp(const GemmFp8Args& a, int parts, float* part, hipStream_t s) {
  constexpr int SMEM = K8Tile<BM>::SMEM;
  auto kern = gemm_fp8_kp_kernel<Tag, BM, TAIL>;
  static thread_local int configured_dev = -1;
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return MLT_ERR_DEVICE;
  if (configured_dev != dev) {
    if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, SMEM) != hipSuccess) {
      (void)hipGetLastError();
      return MLT_ERR_LAUNCH;
    }
    configured_dev = dev;
  }
  const int64_t nbm = (a.M + BM - 1) / BM, nbn = (a.N + 127) / 128;
  const int KT = (int)((a.K + F8_KB - 1) / F8_KB), part_steps = parts > 1 ? (KT + parts - 1) / parts : 0;
  const bool joined = parts == 2 && part_steps < KT;     // (as part_bytes has it)
  if (parts > 1) parts = (KT + part_steps - 1) / part_steps;                // no empty part
  hipLaunchKernelGGL(kern, dim3((unsigned)(nbm * nbn * parts)), dim3(G8_NT), SMEM, s, (int)a.M, (int)a.N, (int)a.K, a.A, a.lda, a.Sa, a.ldsa, a.B, a.ldb, a.Sb, a.ldsb, a.C,
                     a.ldc, (int)nbm, (int)nbn, device_xcds(), part_steps, joined ? 1 : 0, part);
  if (hipGetLastError() != hipSuccess) return MLT_ERR_LAUNCH;
  if (part_steps == 0 || joined) return MLT_OK;
  GemmArgs g{a.M, a.N, a.K, nullptr, 0, nullptr, 0, 1, a.C, a.ldc, a.dtype, GEMM_AUTO, 0};
  g.scratch = part;
  return run_splitk_reduce(g, parts, a.M * a.N, s);
}

template <typename Tag, int BM>
int run_fp8_kp(const GemmFp8Args& a, int parts, float* part, hipStream_t s) {
  return a.K % F8_KB ? launch_fp8_kp<Tag, BM, true>(a, parts, part, s) : launch_fp8_kp<Tag, BM, false>(a, parts, part, s);
}

__global__ void zero_rows_kernel(uint16_t* __restrict__ C, int64_t ldc, int M, int N) {
  for (int64_t e = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; e < (int64_t)M * N; e += (int64_t)gridDim.x * blockDim.x) C[e / N * ldc + e % N] = 0;
}

// Estimated time (us) of a kernel on ncu CUs, fitted to 260 shapes of 65 to 4096 rows (rms of the error 6 %; the choice by it costs 0.6 % on average against
// the best of them): a launch, then rounds of workgroups over the chip, each round its K steps (slower the more of the chip is busy: delivery from the L2s, power) and
// a prologue and epilogue; writing C; with K in parts writing and adding up the partial results.
// us per step and tile: 256 x 256 1.18 to 1.48, 256 x 128 0.79 to 0.91, 128 x 128 0.56 to 0.62 and, two to a CU, 1.09 for both.
// The kernel for few rows (fitted to 1000 shapes of 1 to 4096 rows, rms 10 % up to 64 rows and 7 % above; the choice among all kernels costs 1 % on average): B from memory,
// A and B at what a CU takes, 50 to 130 bytes a ns, A once for each group of columns, and the wavefronts' turns at pieces of K. It wins where a matrix is too small for
// a tile on every CU: 128 x 1024 x 4096 8.1 us, by 128 x 128 tiles and 8 parts of K 13.0; 512 x 512 x 1024 5.0 and 9.5; 1024 x 1024 x 1024 8.7 and 9.7.
double fp8_estimate(int variant, int parts, int64_t M, int64_t N, int64_t K, int64_t ncu) {
  const double mb = (double)M * N * 1e-6;                // of elements of C
  if (variant == GEMM_SKINNY) {
    // as gemm_fp8_skinny.hip lays it out: z rows of workgroups, `rows` of C each; cols columns a workgroup, in groups; rounds of workgroups; what one reads of A and B (KB)
    const int64_t rows = gemm_fp8_skinny_rows(M), z = (M + rows - 1) / rows, per = z * parts, wide = ncu > per ? ncu / per : 1, nwg = N < wide ? N : wide, cols = (N + nwg - 1) / nwg;
    const int64_t cb = gemm_skinny_cols(N, parts, ncu / z), padded = rows <= 4 ? 4 : (rows + 15) / 16 * 16, pieces = ((K + 255) / 256 + parts - 1) / parts;
    const double groups = (double)((cols + (padded <= 32 ? 127 : 63)) / (padded <= 32 ? 128 : 64)), rounds = (double)((nwg * per + ncu - 1) / ncu), nk = (double)N * K * 1e-6;
    const double k = (pieces * 256 < K ? pieces * 256 : K) * 1e-3, a = padded * k, b = (cols + cb - 1) / cb * cb * k, turns = (double)((pieces + 7) / 8), tile = (double)cols * rows;
    if (z == 1)
      return 2.27 + 0.053 * nk + groups * (1.98 + 0.0124 * a + 0.067 * turns) + 0.0142 * b + 0.78 * mb + (parts > 1 ? 0.73 + parts * (0.15 + 3.46 * mb + 1.2e-4 * tile) : 0.0);
    return 3.16 + rounds * (groups * (0.34 + 0.0064 * a + 1.07 * turns) + 0.0218 * b) + 2.96 * mb +
           (parts > 1 ? 1.29 * ((cols * rows + 2047) / 2048) + parts * (0.3 + 1.58 * mb + 1.4e-4 * tile * rounds) : 0.0);
  }
  const int64_t KT = (K + F8_KB - 1) / F8_KB, steps = (KT + parts - 1) / parts;
  auto tiles = [&](int64_t bm, int64_t bn) { return (M + bm - 1) / bm * ((N + bn - 1) / bn) * ((KT + steps - 1) / steps); };
  if (variant == GEMM_128_PP16) {                        // two workgroups per CU; up to ncu of them, one each
    const int64_t w = tiles(128, 128), full = w / (2 * ncu), rest = w % (2 * ncu);
    const int64_t both = full + (rest > ncu ? 1 : 0), one = rest > 0 && rest <= ncu ? 1 : 0;
    return 3.35 + steps * (1.09 * both + 0.77 * one) + 0.28 * (both + one) + 0.38 * mb;
  }
  struct Cost { int64_t bm, bn; double step, fill, launch, round; };
  const Cost c = variant == GEMM_256_PP16 ? Cost{256, 256, 1.18, 0.305, 1.6, 5.6}
               : variant == GEMM_256X128_KP ? Cost{256, 128, 0.79, 0.125, 2.8, 4.8}
               : variant == GEMM_224X128_KP ? Cost{224, 128, 0.75, 0.09, 3.2, 3.7}
               : variant == GEMM_192X128_KP ? Cost{192, 128, 0.69, 0.07, 3.0, 3.6} : Cost{128, 128, 0.56, 0.06, 2.6, 3.3};
  const int64_t w = tiles(c.bm, c.bn), rounds = (w + ncu - 1) / ncu;
  return c.launch + steps * (c.step * rounds + c.fill * w / ncu) + c.round * rounds + 0.3 * mb + (parts == 2 ? 3.2 + 1.65 * mb : parts > 2 ? 2.5 + parts * (0.2 + 1.4 * mb) : 0.0);
}

struct Fp8Plan { int variant, parts; };

int64_t kp_rows_of(int variant) { return variant == GEMM_256X128_KP ? 256 : variant == GEMM_224X128_KP ? 224 : variant == GEMM_192X128_KP ? 192 : 128; }
int64_t kp_tiles(int variant, const GemmFp8Args& a) { return (a.M + kp_rows_of(variant) - 1) / kp_rows_of(variant) * ((a.N + 127) / 128); }
// Bytes of the partial results of a plan with K in parts. Two parts of a tile are joined by the workgroup that comes last (777 x 4096 x 14336: 61.4 us, by a second kernel
// 65.1; 512 x 4096 x 4096 22.8 and 24.1), more by a second kernel (400 x 4096 x 8192 in four 30.5 us, joined 36.0).
int64_t part_bytes(const Fp8Plan& p, const GemmFp8Args& a) {
  if (p.variant == GEMM_SKINNY || p.parts > 2) return p.parts * a.M * a.N * (int64_t)sizeof(float);
  const int64_t floats = p.variant == GEMM_256X128_KP ? K8Tile<256>::PART : p.variant == GEMM_224X128_KP ? K8Tile<224>::PART : p.variant == GEMM_192X128_KP ? K8Tile<192>::PART : K8Tile<128>::PART;
  return p.parts * kp_tiles(p.variant, a) * floats * (int64_t)sizeof(float);
}

Fp8Plan plan_fp8(const GemmFp8Args& a, int max_parts, int64_t ncu) {
  static const int tall[] = {GEMM_256X128_KP, GEMM_224X128_KP, GEMM_192X128_KP, GEMM_128_KP};
  auto known = [&](int v) { return v == GEMM_256_PP16 || v == GEMM_128_PP16 || v == tall[0] || v == tall[1] || v == tall[2] || v == tall[3] || (v == GEMM_SKINNY && a.M <= GEMM_FP8_FEW_ROWS); };
  const int forced = known(a.forced) ? a.forced : GEMM_AUTO;
  Fp8Plan best{forced == GEMM_AUTO ? GEMM_256_PP16 : forced, 1};
  double least = 1e30;
  auto workgroups = [&](int v, int parts) {
    return v == GEMM_256_PP16 ? (a.M + 255) / 256 * ((a.N + 255) / 256) : v == GEMM_128_PP16 ? (a.M + 127) / 128 * ((a.N + 127) / 128) : kp_tiles(v, a) * parts;
  };
  auto offer = [&](int v, int parts) {
    if (forced != GEMM_AUTO && v != forced) return;
    if (v != GEMM_SKINNY && !launch_fits(workgroups(v, parts), G8_NT)) return;
    if (parts == 2 && v != GEMM_SKINNY && kp_tiles(v, a) > kScratchCounters) return;       // a counter for each tile
    if (parts > 1 && a.forced_parts == 0 && part_bytes(Fp8Plan{v, parts}, a) > kStaticScratchBytes) return;
    const double t = fp8_estimate(v, parts, a.M, a.N, a.K, ncu);
    if (t < least) { least = t; best = Fp8Plan{v, parts}; }
  };
  for (int parts = 1; parts <= max_parts; parts *= 2) {
    if (a.forced_parts > 0 ? parts != a.forced_parts && max_parts > 1 : parts > 1 && a.K < 256 * parts) continue;
    for (int v : tall) offer(v, parts);
    if (a.M <= GEMM_FP8_FEW_ROWS) offer(GEMM_SKINNY, parts);
  }
  if (a.forced_parts <= 1 || max_parts == 1 || best.parts == 1) {
    offer(GEMM_256_PP16, 1);
    offer(GEMM_128_PP16, 1);
  }
  if (least < 1e30) return best;
  // nothing that was asked for can be launched: without the parts, then without the kernel
  GemmFp8Args b = a;
  if (a.forced_parts > 1) b.forced_parts = 1;
  else if (forced != GEMM_AUTO) b.forced = GEMM_AUTO;
  else return Fp8Plan{GEMM_AUTO, 0};
  return plan_fp8(b, max_parts, ncu);
}

template <typename Tag>
int run_fp8_t(const GemmFp8Args& a, hipStream_t s, char* name, size_t size) {
  if (a.K == 0) {
    snprintf(name, size, "gemm_fp8_zero");
    hipLaunchKernelGGL(zero_rows_kernel, dim3(1024), dim3(256), 0, s, a.C, a.ldc, (int)a.M, (int)a.N);
    return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
  }
  DeviceInfo di;
  const int64_t ncu = device_info(di) && di.ncu > 0 ? di.ncu : 256;
  Fp8Plan p = plan_fp8(a, 8, ncu);
  if (p.parts == 0) return MLT_ERR_UNSUPPORTED;          // more workgroups than a launch can have, whatever the tile
  float* part = nullptr;
  if (p.parts > 1) {
    part = cached_scratch(part_bytes(p, a), s);
    if (!part) p = plan_fp8(a, 1, ncu);                  // no scratch to be had: the best of the plain forms
  }
  const char* tile = p.variant == GEMM_SKINNY ? "skinny" : p.variant == GEMM_256_PP16 ? "256x256_pp" : p.variant == GEMM_128_PP16 ? "128x128_pp" : p.variant == GEMM_256X128_KP ? "256x128_kp"
                   : p.variant == GEMM_224X128_KP ? "224x128_kp" : p.variant == GEMM_192X128_KP ? "192x128_kp" : "128x128_kp";
  if (p.parts > 1) snprintf(name, size, "gemm_fp8_%s_splitk%d", tile, p.parts);
  else snprintf(name, size, "gemm_fp8_%s", tile);
  switch (p.variant) {
    case GEMM_SKINNY: return run_gemm_fp8_skinny(a, p.parts, part, s);
    case GEMM_256_PP16: return run_fp8_tile<Tag, 256>(a, s);
    case GEMM_128_PP16: return run_fp8_tile<Tag, 128>(a, s);
    case GEMM_256X128_KP: return run_fp8_kp<Tag, 256>(a, p.parts, part, s);
    case GEMM_224X128_KP: return run_fp8_kp<Tag, 224>(a, p.parts, part, s);
    case GEMM_192X128_KP: return run_fp8_kp<Tag, 192>(a, p.parts, part, s);
  }
  return run_fp8_kp<Tag, 128>(a, p.parts, part, s);
}

}  // namespace

int run_gemm_fp8(const GemmFp8Args& a, hipStream_t s, char* name, size_t size) {
  return a.dtype == MLT_BF16 ? run_fp8_t<bf16_tag>(a, s, name, size) : run_fp8_t<f16_tag>(a, s, name, size);
}

}  // namespace mlt
