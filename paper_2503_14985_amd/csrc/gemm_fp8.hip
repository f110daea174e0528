// C = A * B^T on e4m3 operands with a scale for each block of 128 of K (mlt_gemm_fp8):
//   C[m][n] = sum over blocks kb of Sa[kb][m] * Sb[kb][n / 128] * sum over k in kb of A[m][k] * B[n][k]
// One MFMA (16x16x128) multiplies a block's 128 k of a 16 x 16 tile; its fp32 result, started from zero, goes into the fp32
// accumulator with the product of the two scales. That is four fused multiply-adds behind each MFMA of 32 clocks, which take 16 clocks of
// the vector unit beside it: they are issued one MFMA late, while the next one runs.
//
// The schedule is that of gemm_pp.hip, whose K step of 64 16-bit values has the bytes of a K step of 128 here: workgroup tile 256 x 256
// (or 128 x 128, two workgroups per CU), 8 wavefronts as 2 x 4, the two of a SIMD half a step apart, one refilling its
// fragments from LDS while the other multiplies; direct-to-LDS loads into a ring of five operand tiles A_0 B_0 A_1 B_1 A_2 ...,
// group 1 fetching A and group 0 B; 16-byte chunk c of tile row r at position c ^ ((r >> 1) & 7).
// The ring fills the LDS, so the scales of A go through registers: a lane loads one row's scale (of each 64 of its wavefront's rows) for
// the next step, and swaps between lane groups spread a row's scale over the four groups that hold its results (rows of A are the
// columns of the MFMA, so a lane has one row a tile). Those loads sit in front of the step's direct ones, behind a wait for
// all earlier ones: A of the next step has to have landed by the end of that phase anyway, and B has.
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

  // ---- global -> LDS: the wavefronts of group 1 fill the A tiles, those of group 0 the B tiles, NL blocks of 8 rows each. Row and
  // offset of a lane are computed at each load: as registers they would not fit beside accumulators and fragments.
  const char* ld_base = reinterpret_cast<const char*>(grp ? A + (int64_t)m0 * lda : B + (int64_t)n0 * ldb);
  const uint32_t ld_row = (uint32_t)(grp ? lda : ldb);
  const int ld_last = (grp ? M - m0 : N - n0) - 1;       // last row inside the matrix
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lptr_t)smem;
  const bool stream = grp == 1 ? nbn == 1 : nbm == 1;    // (read once: streaming form)
  auto issue_loads = [&](int t, int slot) {
    const char* gp = ld_base + (int64_t)t * F8_KB;
    const uint32_t dst = lds0 + slot * SLOT + (wave & 3) * (NL * 1024);
    int ln = lane;
    asm volatile("" : "+v"(ln));                         // (not hoisted out of the loop)
    const int r0 = (wave & 3) * NL * 8 + (ln >> 3);
    uint32_t voff[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int r = r0 + 8 * i, rr = r < ld_last ? r : ld_last;
      uint32_t c = (uint32_t)((ln & 7) ^ ((r >> 1) & 7)) * 16u;
      if (TAIL && t == KT - 1 && (int)c >= k_tail) c = 0u;   // stays inside the matrix; zeroed in the fragments
      voff[i] = (uint32_t)rr * ld_row + c;
    }
    if (stream) {
#pragma unroll
      for (int i = 0; i < NL; ++i) load_lds16_stream(gp, voff[i], dst + i * 1024);
    } else {
#pragma unroll
      for (int i = 0; i < NL; ++i) load_lds16(gp, voff[i], dst + i * 1024);
    }
  };

  // ---- scales: of row 64 i + lane of this wavefront's rows (with 64 rows: i = 0), and of the block of its columns
  constexpr int NS = WTM / 64;
  int srow[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const int r = m0 + wm * WTM + 64 * i + lane;
    srow[i] = r < M ? r : M - 1;
  }
  const int ncol = n0 + wn * WTN < N ? n0 + wn * WTN : N - 1;
  const float* sb_at = Sb + ncol / F8_KB;
  float sa[NS], sb;
  auto load_scales = [&](int t) {
#pragma unroll
    for (int i = 0; i < NS; ++i) sa[i] = Sa[(int64_t)t * ldsa + srow[i]];
    sb = sb_at[(int64_t)t * ldsb];
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
  auto read_frags = [&](const char* ta, const char* tb) {
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
      for (int i = 0; i < TA; ++i) af[kk][i] = lds_read8<u32x4>(ta, a_off[kk] + i * 16 * F8_KB);
#pragma unroll
      for (int j = 0; j < TB; ++j) bf[kk][j] = lds_read8<u32x4>(tb, b_off[kk] + j * 16 * F8_KB);
    }
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
  issue_loads(0, grp ? 0 : 1);
  if (KT > 1) { issue_loads(1, grp ? 2 : 3); __builtin_amdgcn_s_waitcnt(wait_imm(NL, 0)); }
  else __builtin_amdgcn_s_waitcnt(wait_imm(0, 0));
  MLT_BARRIER();
  if (grp == 1) MLT_BARRIER();

  int slot_a = 0;                                         // slot of A_k; B_k is in the next one
#pragma clang loop unroll(disable)                         // (nor a first iteration peeled off: its copy of the fragments does not fit)
  for (int k = 0; k < KT; ++k) {
    const int slot_b = slot_a + 1 == G8_NSLOT ? 0 : slot_a + 1;
    // ---- memory phase
    read_frags(smem + slot_a * SLOT, smem + slot_b * SLOT);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));          // group 1: A_{k+1}; both: the scales of step k
    __builtin_amdgcn_sched_barrier(0);
    float now[NS];                                        // this step's scales, row by lane
#pragma unroll
    for (int i = 0; i < NS; ++i) now[i] = sa[i] * sb;
    if (k + 1 < KT) load_scales(k + 1);
    __builtin_amdgcn_sched_barrier(0);
    if (grp == 1) {
      if (k + 2 < KT) issue_loads(k + 2, slot_a + 4 >= G8_NSLOT ? slot_a + 4 - G8_NSLOT : slot_a + 4);
    } else {
      if (k >= 1 && k + 1 < KT) issue_loads(k + 1, slot_a + 3 >= G8_NSLOT ? slot_a + 3 - G8_NSLOT : slot_a + 3);
    }
    __builtin_amdgcn_s_waitcnt(wait_imm(63, 0));
    if (TAIL && k == KT - 1) zero_tail();
    MLT_BARRIER();
    __builtin_amdgcn_sched_barrier(0);
    // ---- compute phase
    // (the empty asm statements keep each MFMA and each sum where it is written: behind the last MFMA all parts would be alive)
    f32x4 late;
    float s[4], late_s = 0.f;
#pragma unroll
    for (int e = 0; e <= TA * TB; ++e) {
      f32x4 part;
      if (e < TA * TB) {
        part = mfma16_e4m3(bf[0][e % TB], bf[1][e % TB], af[0][e / TB], af[1][e / TB], f32x4{0.f, 0.f, 0.f, 0.f});
        asm volatile("" : "+v"(part));
        __builtin_amdgcn_sched_barrier(0);
        if (e % (4 * TB) == 0) spread_groups(now[e / (4 * TB)], s);
      }
      if (e > 0) {
        f32x4& to = acc[(e - 1) / TB][(e - 1) % TB];
#pragma unroll
        for (int r = 0; r < 4; ++r) to[r] += late[r] * late_s;
        asm volatile("" : "+v"(to));
      }
      late = part;
      late_s = s[e / TB % 4];
      __builtin_amdgcn_sched_barrier(0);
    }
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

template <typename Tag, int BT, bool TAIL>
int launch_fp8(const GemmFp8Args& a, hipStream_t s) {
  constexpr int SMEM = G8Tile<BT>::SMEM;
  auto kern = gemm_fp8_kernel<Tag, BT, TAIL>;
  static thread_local int configured_dev = -1;          // opt in to > 64 KB LDS once per device
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return MLT_ERR_DEVICE;
  if (configured_dev != dev) {
    if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, SMEM) != hipSuccess) {
      (void)hipGetLastError();
      return MLT_ERR_LAUNCH;
    }
    configured_dev = dev;
  }
  const int64_t nbm = (a.M + BT - 1) / BT, nbn = (a.N + BT - 1) / BT;
  if (nbm * nbn > 0x7fffffff) return MLT_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(kern, dim3((unsigned)(nbm * nbn)), dim3(G8_NT), SMEM, s, (int)a.M, (int)a.N, (int)a.K, a.A, a.lda, a.Sa, a.ldsa, a.B, a.ldb, a.Sb, a.ldsb, a.C,
                     a.ldc, (int)nbm, (int)nbn, device_xcds());
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

template <typename Tag, int BT>
int run_fp8_tile(const GemmFp8Args& a, hipStream_t s) {
  return a.K % F8_KB ? launch_fp8<Tag, BT, true>(a, s) : launch_fp8<Tag, BT, false>(a, s);
}

__global__ void zero_rows_kernel(uint16_t* __restrict__ C, int64_t ldc, int M, int N) {
  for (int64_t e = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; e < (int64_t)M * N; e += (int64_t)gridDim.x * blockDim.x) C[e / N * ldc + e % N] = 0;
}

template <typename Tag>
int run_fp8_t(const GemmFp8Args& a, hipStream_t s, const char** name) {
  if (a.K == 0) {
    *name = "gemm_fp8_zero";
    hipLaunchKernelGGL(zero_rows_kernel, dim3(1024), dim3(256), 0, s, a.C, a.ldc, (int)a.M, (int)a.N);
    return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
  }
  DeviceInfo di;
  const int64_t ncu = device_info(di) && di.ncu > 0 ? di.ncu : 256;
  if (a.M <= 64) {
    int parts = a.forced_parts > 1 ? a.forced_parts : 1;
    float* part = nullptr;
    if (parts > 1) {
      part = cached_scratch(parts * a.M * a.N * (int64_t)sizeof(float), s);
      if (!part) parts = 1;
    }
    static const char* const names[9] = {"", "gemm_fp8_skinny", "gemm_fp8_skinny_splitk2", "", "gemm_fp8_skinny_splitk4", "", "", "", "gemm_fp8_skinny_splitk8"};
    *name = names[parts];
    return run_gemm_fp8_skinny(a, parts, part, s);
  }
  const int64_t big = ((a.M + 255) / 256) * ((a.N + 255) / 256);
  if (big >= ncu) {
    *name = "gemm_fp8_256x256";
    return run_fp8_tile<Tag, 256>(a, s);
  }
  *name = "gemm_fp8_128x128";
  return run_fp8_tile<Tag, 128>(a, s);
}

}  // namespace

int run_gemm_fp8(const GemmFp8Args& a, hipStream_t s, const char** name) {
  return a.dtype == MLT_BF16 ? run_fp8_t<bf16_tag>(a, s, name) : run_fp8_t<f16_tag>(a, s, name);
}

}  // namespace mlt
