// Quantisation to e4m3 with a scale for each block of 128 columns, of one row (activations) or of 128 rows (a weight): what
// mlt_gemm_fp8 multiplies. q = rne(x / s), s the smallest power of two with max |x| <= 448 s (fp8.h).
//
// Bound by memory: 2 bytes read and 1 written an element, each once. A lane holds 8 neighbouring elements (16 bytes), 16 lanes a
// block's row of 256 bytes; the maximum of a row's block is four DPP steps away, that of 128 rows another exchange through LDS.
#include <type_traits>

#include "fp8.h"
#include "mlt_internal.h"

namespace mlt {

namespace {

constexpr int QT_NT = 256;

// maximum over the 16 lanes of a row; every lane gets it
__device__ __forceinline__ float row16_max(float x) {
  auto step = [&](auto ctrl) __attribute__((always_inline)) {
    x = __builtin_fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, false)));
  };
  step(std::integral_constant<int, 0xB1>{});     // quad_perm [1,0,3,2]
  step(std::integral_constant<int, 0x4E>{});     // quad_perm [2,3,0,1]
  step(std::integral_constant<int, 0x141>{});    // row_half_mirror
  step(std::integral_constant<int, 0x140>{});    // row_mirror
  return x;
}

template <typename Tag>
__device__ __forceinline__ float max8(const u32x4& v) {
  float x[8];
  unpack8<Tag>(v, x);
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = __builtin_fmaxf(m, finite_abs(x[e]));
  return m;
}
template <typename Tag>
__device__ __forceinline__ u32x2 quant8(const u32x4& v, float inv) {
  float x[8];
  unpack8<Tag>(v, x);
  return u32x2{to_e4m3x4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv), to_e4m3x4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv)};
}

// A workgroup takes 4 * RPW rows and 4 blocks of columns, a wavefront RPW rows of them.
template <typename Tag, int RPW>
__global__ __launch_bounds__(QT_NT) void quant_rows_kernel(int M, int K, const uint16_t* __restrict__ X, int64_t ldx,
                                                           uint8_t* __restrict__ Xq, int64_t ldq, float* __restrict__ S, int64_t lds) {
  __shared__ float sc[4][4 * RPW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row0 = (int)blockIdx.y * 4 * RPW, col = (int)blockIdx.x * 512 + lane * 8;
  const bool in = col < K;
  u32x4 v[RPW];
#pragma unroll
  for (int i = 0; i < RPW; ++i) {
    const int r = row0 + wave * RPW + i;
    v[i] = u32x4{0u, 0u, 0u, 0u};
    if (in && r < M) v[i] = load_stream16(X + (int64_t)r * ldx + col);
  }
#pragma unroll
  for (int i = 0; i < RPW; ++i) {
    const int r = row0 + wave * RPW + i;
    const float s = pow2_scale(row16_max(max8<Tag>(v[i])));
    if (in && r < M) *reinterpret_cast<u32x2_mem*>(Xq + (int64_t)r * ldq + col) = quant8<Tag>(v[i], pow2_inv(s));
    if ((lane & 15) == 0) sc[lane >> 4][wave * RPW + i] = s;
  }
  __syncthreads();
  for (int e = tid; e < 16 * RPW; e += QT_NT) {
    const int kb = (int)blockIdx.x * 4 + e / (4 * RPW), r = row0 + e % (4 * RPW);
    if (r < M && kb * F8_KB < K) S[(int64_t)kb * lds + r] = sc[e / (4 * RPW)][e % (4 * RPW)];
  }
}

// A workgroup takes a block of 128 x 128, a wavefront 32 rows of it.
template <typename Tag>
__global__ __launch_bounds__(QT_NT) void quant_tiles_kernel(int M, int K, const uint16_t* __restrict__ X, int64_t ldx,
                                                            uint8_t* __restrict__ Xq, int64_t ldq, float* __restrict__ S, int64_t lds) {
  __shared__ float top[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row0 = (int)blockIdx.y * 128 + wave * 32 + (lane >> 4), col = (int)blockIdx.x * F8_KB + (lane & 15) * 8;
  const bool in = col < K;
  u32x4 v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = u32x4{0u, 0u, 0u, 0u};
    if (in && row0 + 4 * i < M) v[i] = load_stream16(X + (int64_t)(row0 + 4 * i) * ldx + col);
  }
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = __builtin_fmaxf(m, max8<Tag>(v[i]));
  m = row16_max(m);
  m = __builtin_fmaxf(m, __shfl_xor(m, 16));
  m = __builtin_fmaxf(m, __shfl_xor(m, 32));
  if (lane == 0) top[wave] = m;
  __syncthreads();
  const float s = pow2_scale(__builtin_fmaxf(__builtin_fmaxf(top[0], top[1]), __builtin_fmaxf(top[2], top[3])));
  const float inv = pow2_inv(s);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (in && row0 + 4 * i < M) *reinterpret_cast<u32x2_mem*>(Xq + (int64_t)(row0 + 4 * i) * ldq + col) = quant8<Tag>(v[i], inv);
  if (tid == 0) S[(int64_t)blockIdx.x * lds + blockIdx.y] = s;
}

template <typename Tag>
int run_quant_t(const QuantArgs& a, hipStream_t s) {
  const unsigned kb = (unsigned)((a.K + F8_KB - 1) / F8_KB);
  if (a.block_rows == 1) {
    constexpr int RPW = 4;
    hipLaunchKernelGGL((quant_rows_kernel<Tag, RPW>), dim3((kb + 3) / 4, (unsigned)((a.M + 4 * RPW - 1) / (4 * RPW))), dim3(QT_NT), 0, s, (int)a.M, (int)a.K,
                       a.X, a.ldx, a.Xq, a.ldq, a.S, a.lds);
  } else {
    hipLaunchKernelGGL((quant_tiles_kernel<Tag>), dim3(kb, (unsigned)((a.M + 127) / 128)), dim3(QT_NT), 0, s, (int)a.M, (int)a.K, a.X, a.ldx, a.Xq, a.ldq, a.S, a.lds);
  }
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

}  // namespace

int run_quant(const QuantArgs& a, hipStream_t s) { return a.dtype == MLT_BF16 ? run_quant_t<bf16_tag>(a, s) : run_quant_t<f16_tag>(a, s); }

}  // namespace mlt
