// e4m3 (OCP: 1 sign, 4 exponent, 3 mantissa bits, largest 448, no infinities) on gfx950: conversions, the scale of a block, the
// MFMA on it. A block's scale is the smallest power of two s with max |x| <= 448 s: x / s is then exact, the only rounding is
// the one to e4m3, and a value that is scaled up by a power of two again loses nothing but what falls below e4m3's
// smallest step. Infinities and NaN do not count for the maximum and become NaN.
#pragma once

#include "mlt_common.h"

namespace mlt {

constexpr int F8_KB = 128;                 // k values of a scale block
typedef __attribute__((ext_vector_type(8))) int i32x8;

// 2^e with e in -100 .. 120, from the maximum of |x| over finite x (a non-negative finite float)
__device__ __forceinline__ float pow2_scale(float amax) {
  const int bits = __builtin_bit_cast(int, amax);
  int e = (bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);       // 448 = 1.75 * 2^8; biased exponent of the scale
  e = e < 27 ? 27 : e;
  return __builtin_bit_cast(float, e << 23);
}
// the smallest power of two >= s in 2^-100 .. 2^126, whose inverse is a normal number (anything that is no positive number: the lower end)
__device__ __forceinline__ float pow2_ceil(float s) {
  if (!(s > 0.f)) return __builtin_bit_cast(float, 27 << 23);
  const int bits = __builtin_bit_cast(int, s);
  int e = (bits >> 23) + ((bits & 0x7fffff) ? 1 : 0);
  e = e < 27 ? 27 : e > 253 ? 253 : e;
  return __builtin_bit_cast(float, e << 23);
}
// 1 / s of a power of two of either range: a power of two as well
__device__ __forceinline__ float pow2_inv(float s) { return __builtin_bit_cast(float, (254 << 23) - __builtin_bit_cast(int, s)); }
// |x| of a finite x, else 0
__device__ __forceinline__ float finite_abs(float x) {
  const float a = __builtin_fabsf(x);
  return a < __builtin_inff() ? a : 0.f;
}

// four values to e4m3, round-to-nearest-even; what overflows, infinities and NaN become NaN
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}
// the four values of a dword
__device__ __forceinline__ f32x4 from_e4m3x4(uint32_t w) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return f32x4{lo[0], lo[1], hi[0], hi[1]};
}
// two of them (the upper two with HI) as a packed pair of the 16-bit type: exact
template <typename Tag, bool HI> __device__ __forceinline__ uint32_t e4m3_pair(uint32_t w);
template <> __device__ __forceinline__ uint32_t e4m3_pair<f16_tag, false>(uint32_t w) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false)); }
template <> __device__ __forceinline__ uint32_t e4m3_pair<f16_tag, true>(uint32_t w) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true)); }
template <> __device__ __forceinline__ uint32_t e4m3_pair<bf16_tag, false>(uint32_t w) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false)); }
template <> __device__ __forceinline__ uint32_t e4m3_pair<bf16_tag, true>(uint32_t w) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true)); }

// the eight values of a 16-byte piece of the 16-bit type
template <typename Tag>
__device__ __forceinline__ void unpack8(const u32x4& v, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = Elem<Tag>::to_f32((uint16_t)(v[e >> 1] >> (16 * (e & 1))));
}

// D(16x16) = A(16x128) * B(128x16) + C on e4m3. A lane supplies 32 of the 128 k values of row (column) l % 16; lanes 16 g ..
// 16 g + 15 have the same ones in both operands, in whatever order they are taken. D as in mfma16.
// The sum is less exact than that of the 16-bit MFMAs: the 8 products of 8 neighbouring bytes are added in fixed point with 13 bits below the leading bit of the
// largest (what lies below is cut off), the groups' sums then in fp32 (measured: beside a product of 2^16 one of 2^3 counts in its group, one of 7 does not;
// in another group all do down to 2^-7). On normal data that is 1e-4 of a result, half of what the rounding to fp16 costs; the exact way, on the 16-bit MFMA, has half the rate.
__device__ __forceinline__ f32x4 mfma16_e4m3(const u32x4& a0, const u32x4& a1, const u32x4& b0, const u32x4& b1, f32x4 c) {
  const i32x8 a = {(int)a0[0], (int)a0[1], (int)a0[2], (int)a0[3], (int)a1[0], (int)a1[1], (int)a1[2], (int)a1[3]};
  const i32x8 b = {(int)b0[0], (int)b0[1], (int)b0[2], (int)b0[3], (int)b1[0], (int)b1[1], (int)b1[2], (int)b1[3]};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
}

// A dword per lane (uniform base + per-lane byte offset) straight into LDS at lds_addr + 4 * lane: load_lds16 of mlt_common.h in the narrow form
__device__ __forceinline__ void load_lds4(const void* base, uint32_t voff, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(lds_addr), "v"(voff), "s"(base) : "memory", "m0");
}
// the same from an address of each lane's own
__device__ __forceinline__ void load_lds4(const void* p, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(lds_addr), "v"(p) : "memory", "m0");
}

}  // namespace mlt
