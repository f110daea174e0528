// Quantisation to e4m3 with a scale for each block of 128 columns, of one row (activations) or of 128 rows (a weight): what
// mlt_gemm_fp8 multiplies. q = rne(x / s), s the smallest power of two with max |x| <= 448 s (fp8.h).
//
// Bound by memory: 2 bytes read and 1 written an element, each once. A lane holds 8 neighbouring elements (16 bytes), 16 lanes a
// block's row of 256 bytes; the maximum of a row's block is four DPP steps away, that of 128 rows another exchange through LDS.
// What lies past the last row or column is read as the last row, the last 8 columns: in the same block, so the maximum is the same, and no load waits for a branch
// (with branches the rows in flight were one 32-register value to the compiler, copied about: 250 registers).
// Measured: rows 8192 x 14336 61 us (5.8 TB/s), 16 x 4096 3.4 us, a launch; 128 x 128 of 14336 x 4096 30 us (5.8 TB/s; blocks of 256 or 512 columns at once, or an
// XCD's workgroups side by side, gave 29 to 34), 256 x 512 3.9 us.
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

// Largest finite |x| of 16-bit numbers, two at a time as integers: |x| plus the distance from infinity to 2^15 is a positive int16 where x is finite and a
// negative one where it is not. (As floats the compiler keeps all of them unpacked for the second pass: 236 registers, half the rate.)
typedef __attribute__((ext_vector_type(2))) short i16x2;
template <typename Tag> constexpr uint32_t ABOVE = std::is_same<Tag, f16_tag>::value ? 0x04000400u : 0x00800080u;
template <typename Tag>
__device__ __forceinline__ i16x2 max8(i16x2 m, const u32x4& v) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    m = __builtin_elementwise_max(m, __builtin_bit_cast(i16x2, v[i] & 0x7FFF7FFFu) + __builtin_bit_cast(i16x2, ABOVE<Tag>));
  return m;
}
template <typename Tag>
__device__ __forceinline__ float top_of(i16x2 m) {
  const int top = m[0] > m[1] ? m[0] : m[1];
  return Elem<Tag>::to_f32((uint16_t)(top - (int)(ABOVE<Tag> & 0xFFFFu)));
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
                                                           uint8_t* __restrict__ Xq, int64_t ldq, float* __restrict__ S, int64_t lds, int nbx) {
  __shared__ float sc[4][4 * RPW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int by = (int)blockIdx.x / nbx, bx = (int)blockIdx.x - by * nbx;
  const int row0 = by * 4 * RPW, col = bx * 512 + lane * 8;
  const bool in = col < K;
  u32x4 v[RPW];
  const uint16_t* x = X + (in ? col : K - 8);
#pragma unroll
  for (int i = 0; i < RPW; ++i) {
    const int r = row0 + wave * RPW + i;
    v[i] = load_stream16(x + (int64_t)(r < M ? r : M - 1) * ldx);
  }
#pragma unroll
  for (int i = 0; i < RPW; ++i) {
    const int r = row0 + wave * RPW + i;
    const float s = pow2_scale(row16_max(top_of<Tag>(max8<Tag>(__builtin_bit_cast(i16x2, ABOVE<Tag>), v[i]))));
    if (in && r < M) *reinterpret_cast<u32x2_mem*>(Xq + (int64_t)r * ldq + col) = quant8<Tag>(v[i], pow2_inv(s));
    if ((lane & 15) == 0) sc[lane >> 4][wave * RPW + i] = s;
  }
  __syncthreads();
  for (int e = tid; e < 16 * RPW; e += QT_NT) {
    const int kb = bx * 4 + e / (4 * RPW), r = row0 + e % (4 * RPW);
    if (r < M && kb * F8_KB < K) S[(int64_t)kb * lds + r] = sc[e / (4 * RPW)][e % (4 * RPW)];
  }
}

// A workgroup takes a block of 128 x 128, a wavefront 32 rows of it.
template <typename Tag>
__global__ __launch_bounds__(QT_NT) void quant_tiles_kernel(int M, int K, const uint16_t* __restrict__ X, int64_t ldx,
                                                            uint8_t* __restrict__ Xq, int64_t ldq, float* __restrict__ S, int64_t lds, int nbx) {
  __shared__ float top[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int by = (int)blockIdx.x / nbx, bx = (int)blockIdx.x - by * nbx;
  const int row0 = by * 128 + wave * 32 + (lane >> 4), col = bx * F8_KB + (lane & 15) * 8;
  const bool in = col < K;
  u32x4 v[8];
  const uint16_t* x = X + (in ? col : K - 8);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = load_stream16(x + (int64_t)(row0 + 4 * i < M ? row0 + 4 * i : M - 1) * ldx);
  i16x2 most = __builtin_bit_cast(i16x2, ABOVE<Tag>);
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max8<Tag>(most, v[i]);
  float m = row16_max(top_of<Tag>(most));
  m = __builtin_fmaxf(m, __shfl_xor(m, 16));
  m = __builtin_fmaxf(m, __shfl_xor(m, 32));
  if (lane == 0) top[wave] = m;
  __syncthreads();
  const float s = pow2_scale(__builtin_fmaxf(__builtin_fmaxf(top[0], top[1]), __builtin_fmaxf(top[2], top[3])));
  const float inv = pow2_inv(s);
#pragma unroll
  for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(v[i]));               // (unpacked after the barrier, not before)
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (in && row0 + 4 * i < M) *reinterpret_cast<u32x2_mem*>(Xq + (int64_t)(row0 + 4 * i) * ldq + col) = quant8<Tag>(v[i], inv);
  if (tid == 0) S[(int64_t)bx * lds + by] = s;
}

template <typename Tag>
int run_quant_t(const QuantArgs& a, hipStream_t s) {
  constexpr int RPW = 4;
  const int64_t cols = a.block_rows == 1 ? 512 : F8_KB, rows = a.block_rows == 1 ? 4 * RPW : 128, nbx = (a.K + cols - 1) / cols, wgs = nbx * ((a.M + rows - 1) / rows);
  if (!launch_fits(wgs, QT_NT)) return MLT_ERR_UNSUPPORTED;
  if (a.block_rows == 1)
    hipLaunchKernelGGL((quant_rows_kernel<Tag, RPW>), dim3((unsigned)wgs), dim3(QT_NT), 0, s, (int)a.M, (int)a.K, a.X, a.ldx, a.Xq, a.ldq, a.S, a.lds, (int)nbx);
  else
    hipLaunchKernelGGL((quant_tiles_kernel<Tag>), dim3((unsigned)wgs), dim3(QT_NT), 0, s, (int)a.M, (int)a.K, a.X, a.ldx, a.Xq, a.ldq, a.S, a.lds, (int)nbx);
  return hipGetLastError() == hipSuccess ? MLT_OK : MLT_ERR_LAUNCH;
}

}  // namespace

int run_quant(const QuantArgs& a, hipStream_t s) { return a.dtype == MLT_BF16 ? run_quant_t<bf16_tag>(a, s) : run_quant_t<f16_tag>(a, s); }

}  // namespace mlt
