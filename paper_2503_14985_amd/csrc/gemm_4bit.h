// What the two kernels of mlt_gemm_w4 share (gemm_4bit.hip, gemm_4bit_tile.hip).
#pragma once
#include "fp8.h"
#include "mlt_common.h"

namespace mlt {

// a 16-bit (8-bit) number for each lane (uniform base + per-lane byte offset), as a dword to lds_addr + 4 * lane
__device__ __forceinline__ void load_lds_u16(const void* base, uint32_t voff, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ushort %1, %2" : : "s"(lds_addr), "v"(voff), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void load_lds_u8(const void* base, uint32_t voff, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ubyte %1, %2" : : "s"(lds_addr), "v"(voff), "s"(base) : "memory", "m0");
}

// 16 + q of nibbles i and i + 4. The two constants are given in registers: and-or takes no two literals.
template <typename Tag> struct Nibbles {
  static constexpr bool BF = __is_same(Tag, bf16_tag);
  static constexpr uint32_t MASK = BF ? 0x00780078u : 0x03c003c0u, SIXTEEN = BF ? 0x41804180u : 0x4c004c00u;
  static __device__ __forceinline__ uint32_t get(uint32_t w, int i, uint32_t mask, uint32_t sixteen) {
    const int right = 4 * i - (BF ? 3 : 6);
    return ((right < 0 ? w << -right : w >> right) & mask) | sixteen;
  }
};

struct W4 {
  int M, N, K, share, rest, lda, ldw;          // share, rest: units of columns (blocks of 16) of every workgroup, and one more for the first ones
  const uint16_t* A;
  const uint8_t* W;
  const uint16_t* S;
  const uint8_t* Z;
  int64_t lds, ldz;                            // (below 2^26)
  uint16_t* C;
  int64_t ldc;
  float* part;
  uint32_t* counter;
};

// Rows m0 .. m0 + M - 1, columns c0 .. c1 - 1 of C: the sums of the parts, in their order (4 elements of a thread at a time, 8 parts of each requested before the first is used).
template <typename Tag, int NT> __device__ __forceinline__ void w4_add_parts(const W4& a, int parts, int m0, int M, int c0, int c1) {
  const int cols = c1 - c0;
  const int64_t part_size = (int64_t)a.M * a.N;
  constexpr int EB = 4;
  for (int e0 = threadIdx.x; e0 < M * cols; e0 += EB * NT) {
    float sum[EB];
    int64_t at[EB];
#pragma unroll
    for (int i = 0; i < EB; ++i) {
      const int e = e0 + i * NT < M * cols ? e0 + i * NT : e0;
      at[i] = (int64_t)(m0 + e / cols) * a.N + c0 + e % cols;
      sum[i] = 0.f;
    }
    for (int p0 = 0; p0 < parts; p0 += 8) {
      float v[8][EB];
#pragma unroll
      for (int p = 0; p < 8; ++p)
        if (p0 + p < parts) {
#pragma unroll
          for (int i = 0; i < EB; ++i) v[p][i] = load_shared(a.part + (p0 + p) * part_size + at[i]);
        }
#pragma unroll
      for (int p = 0; p < 8; ++p)
        if (p0 + p < parts) {
#pragma unroll
          for (int i = 0; i < EB; ++i) sum[i] += v[p][i];
        }
    }
#pragma unroll
    for (int i = 0; i < EB; ++i)
      if (e0 + i * NT < M * cols) {
        const int e = e0 + i * NT;
        a.C[(int64_t)(m0 + e / cols) * a.ldc + c0 + e % cols] = Elem<Tag>::from_f32(sum[i]);
      }
  }
}

// Scales and zero points of a chunk of 128 (gemm_4bit_tile.hip): lanes 16 g .. 16 g + 15 of a wavefront load those of its group w4t_group(g), lanes to spare those of its last group again, where the
// matrix has that group. The last chunk of a row may have fewer (K is a multiple of 32): a group that is not there is not read, whichever lanes would read it.
template <int G> __host__ __device__ __forceinline__ constexpr int w4t_group(int g) { return g < 128 / G ? g : 128 / G - 1; }
template <int G> __host__ __device__ __forceinline__ constexpr bool w4t_group_there(int k0, int g, int last_group) { return k0 / G + w4t_group<G>(g) <= last_group; }

// gemm_4bit_tile.hip: nwg workgroups of up to 8 or 16 blocks of 16 columns for every 64 rows and each part of K
constexpr int W4T_ROWS = 64;
int run_w4_tile(const W4& a, int dtype, int group, int blocks, unsigned nwg, int parts, hipStream_t s);

}  // namespace mlt
