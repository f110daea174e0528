/*
 * mlt — tile-based dense kernels for AMD MI355X (gfx950, CDNA4, wave64), C ABI.
 *
 * The two operations are the dense workloads that arXiv 2503.14985 ("ML-Triton") lowers
 * workgroup -> warp -> intrinsic: a 16-bit GEMM with 32-bit accumulation (Section 2, Listing 1)
 * and a FlashAttention-2-style attention forward (Section 2.5, Algorithm 1). Here both are
 * hand-written HIP kernels; the workgroup tile -> per-wavefront sub-tile -> MFMA tile split is
 * fixed at compile time per kernel variant.
 *
 * Conventions shared by every entry point
 *   - All data pointers are DEVICE pointers to memory the caller owns. The library never frees
 *     or keeps them. Inputs and outputs must not overlap.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream). Work is enqueued
 *     asynchronously on it; no entry point synchronises the device.
 *   - `dtype` selects the 16-bit element type of every input and output tensor:
 *     MLT_BF16 (bfloat16) or MLT_FP16 (IEEE binary16). Accumulation is fp32; outputs are
 *     rounded to `dtype` with round-to-nearest-even.
 *   - Return value: MLT_OK or a negative mlt_status. No C++ exception crosses the boundary and
 *     nothing aborts. On an error nothing has been enqueued.
 *     The 8-bit operators say themselves which of their tensors are e4m3 or fp32.
 *   - Device memory of the library's own: the GEMM entry points (few tiles against a long K),
 *     mlt_paged_attn_decode and its 8-bit form (few sequences x heads), mlt_mha_fwd and the attention of packed sequences and prompts (few query tiles against many
 *     keys) and mlt_paged_attn_decode_prefix (unless it is given `work`) may spread one result over several workgroups and then keep fp32 partial results in a
 *     scratch buffer, one per (device, stream), allocated with hipMalloc at the first call that
 *     needs it, grown by doubling from 4 MiB (64 MiB covers every split the library chooses by
 *     itself, but for shared prefixes of very large batches) and kept until the process ends. Calls on one stream are ordered by the stream, whichever threads make them; calls
 *     on different streams use different buffers (on hipStreamPerThread: of different threads). If the allocation fails, or the stream is
 *     recording into a graph (which may be replayed at any time and on any stream, so that it must
 *     not share the stream's buffer), the call runs without the split (same result up to summation
 *     order). mlt_gemm_noalloc never allocates.
 */
#ifndef MLT_H_
#define MLT_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { MLT_BF16 = 0, MLT_FP16 = 1 } mlt_dtype;

typedef enum {
  MLT_OK = 0,
  MLT_ERR_INVALID_ARG = -1, /* null pointer, negative size, leading dimension too small, bad dtype */
  MLT_ERR_UNSUPPORTED = -2, /* valid request with no kernel (e.g. head dimension not 64 or 128; sizes that would take a launch of more
                               than 2^32 work-items, some 10^7 workgroups) */
  MLT_ERR_LAUNCH = -3,      /* the HIP runtime rejected the kernel launch */
  MLT_ERR_DEVICE = -4,      /* no usable gfx950 device is current */
  MLT_ERR_SCRATCH = -5      /* mlt_gemm_noalloc: the call needs more than the fixed scratch array holds */
} mlt_status;

/*
 * GEMM, Section 2 of the paper (A is m x k, B is k x n, C is m x n; 16-bit inputs, fp32
 * accumulate as in Listing 1). Computes C = A * B, overwriting C (no accumulation into the
 * previous contents), output rounded to `dtype`.
 *
 *   A      device, M x K row-major, row stride lda >= K elements
 *   B      device; transB == 0: K x N row-major, row stride ldb >= N
 *                  transB != 0: the N x K row-major array holding B transposed (B in
 *                               column-major order), row stride ldb >= K
 *   C      device, M x N row-major, row stride ldc >= N; written, never read
 *
 * M, N or K may be 0: M == 0 or N == 0 is a no-op, K == 0 stores zeros. Any positive shape and
 * any leading dimensions/alignments are accepted; shapes and pointers that allow 16-byte vector
 * access (K, N, lda, ldb multiples of 8 and 16-byte aligned bases) take the fastest kernels, others
 * forms of the tile kernels for any alignment, with identical results up to summation order.
 */
int mlt_gemm(int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const void* B,
             int64_t ldb, int transB, void* C, int64_t ldc, int dtype, void* stream);

/*
 * mlt_gemm for callers that cannot allocate device memory: code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc. Same arguments, same kernels and the same
 * result, bit for bit, as mlt_gemm on a stream that is not recording (there mlt_gemm leaves the
 * split out, see above). Where mlt_gemm splits K across workgroups (few tiles against
 * a long K) and keeps the fp32 partial products in a scratch buffer it allocates, this entry point
 * keeps them in a fixed array of 32 MiB in device memory that is part of the library (one copy
 * per GPU the library runs on, held until the process ends). It calls no hipMalloc, hipFree or
 * other allocating routine. The library's own choice of a split never needs more than that;
 * a split forced through mlt_diag_force_k_parts that needs more than 32 MiB (parts * M * N * 4
 * bytes) is refused with MLT_ERR_SCRATCH and nothing is enqueued. All calls on one GPU share that
 * GPU's array: two calls of this entry point that may run at the same time on one GPU (different
 * streams) race; calls on one stream, and calls on different GPUs, do not.
 */
int mlt_gemm_noalloc(int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const void* B,
                     int64_t ldb, int transB, void* C, int64_t ldc, int dtype, void* stream);

/*
 * The paper's own form of the GEMM (Section 2, Listing 1): C += A * B with C in fp32, i.e. the
 * fp32 accumulator is added to what C already holds and nothing is rounded to 16 bit.
 * A, B, transB, dtype as for mlt_gemm; C is device, M x N row-major fp32, row stride ldc >= N
 * (in fp32 elements), 4-byte aligned, read and written. M, N or K equal to 0 is a no-op. The
 * read-modify-write of C is not atomic: do not run two calls on the same C concurrently.
 */
int mlt_gemm_acc(int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const void* B,
                 int64_t ldb, int transB, float* C, int64_t ldc, int dtype, void* stream);

/*
 * mlt_gemm with the paper's `tiling` hint (Section 3.1, "Compiler Hint"): how the wavefronts of a
 * workgroup divide its 256 x 256 output tile. All settings compute the same C (up to summation
 * order) and obey the same tolerances; what changes is the kernel.
 *   tiling 0  the library's choice (the same as mlt_gemm)
 *          1  horizontal: evenly along the rows only, 8 wavefronts x (32 x 256)
 *          2  vertical: evenly along the columns only, 8 wavefronts x (256 x 32)
 *          3  square: 2 x 2 wavefronts x (128 x 128)
 * The hint applies to operands that allow 16-byte vector access (see mlt_gemm); others are
 * treated as with tiling 0, K = 0 stores zeros, and the skinny kernel (M <= 64 with B stored N x K)
 * and the smaller workgroup tiles of small aligned problems are chosen only for tiling 0. Returns as
 * mlt_gemm; MLT_ERR_INVALID_ARG also for an unknown `tiling`.
 */
int mlt_gemm_tiled(int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const void* B,
                   int64_t ldb, int transB, void* C, int64_t ldc, int dtype, int tiling,
                   void* stream);

/*
 * GEMM with a fused epilogue, C = act(A*B + bias): the post-operation fusion the paper expects to
 * fall out of its layout propagation from the root operation (Section 3.1, the remark on pre- and
 * post-operation fusion), here written into the kernels' epilogues. Arguments as for mlt_gemm,
 * plus
 *   bias   device, N elements of `dtype` added to every row of A*B in fp32 before the activation,
 *          or NULL for none; only read
 *   act    0 none, 1 ReLU max(x, 0), 2 GELU in its exact form x * Phi(x) = x/2 * (1 + erf(x/sqrt 2))
 * The fp32 accumulator plus bias goes through the activation in fp32 and is rounded once (RNE) to
 * the 16-bit C. K = 0 gives C = act(bias) (act(0) without a bias). Returns as mlt_gemm;
 * MLT_ERR_INVALID_ARG also for an unknown `act` or a misaligned bias.
 */
int mlt_gemm_bias_act(int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const void* B,
                      int64_t ldb, int transB, const void* bias, int act, void* C, int64_t ldc,
                      int dtype, void* stream);

/*
 * Attention forward, Section 2.5 / Algorithm 1 of the paper, per batch b and head h:
 *   O = softmax(scale * Q K^T  [+ causal mask]) V
 * computed tile by tile with the online-softmax recurrence (running row maximum m and row sum
 * l in fp32, P rounded to `dtype` before the second product, one division by l at the end).
 *
 *   Q, O   device, contiguous [B, H, Sq, D], D innermost
 *   K, V   device, contiguous [B, H, Sk, D]
 *   causal != 0: key j is visible to query i iff j <= i (lower triangle including the
 *                diagonal, aligned at the top-left corner; key 0 is visible to every query).
 *
 * D must be 64 or 128 and one head's K must stay below 2 GiB (Sk * D * 2 < 2^31), else
 * MLT_ERR_UNSUPPORTED. B, H or Sq equal to 0 is a no-op. Sk must be >= 1 (a softmax over no keys
 * is undefined: MLT_ERR_INVALID_ARG). All four base pointers must be 16-byte aligned and scale
 * must be finite (MLT_ERR_INVALID_ARG otherwise).
 */
int mlt_mha_fwd(int64_t B, int64_t H, int64_t Sq, int64_t Sk, int64_t D, const void* Q,
                const void* K, const void* V, void* O, float scale, int causal, int dtype,
                void* stream);

/*
 * Paged attention for decoding, Section 3.2 of the paper: ONE query per (sequence b, head h) over
 * the seq_lens[b] keys and values of that sequence, which live in fixed-size blocks of a cache:
 *   o = sum_j softmax_j(scale * q . k_j) v_j,   j = 0 .. seq_lens[b] - 1.
 * The keys are split over the wavefronts of a workgroup and the partial maxima, sums and outputs
 * are reduced through LDS (the paper's warp-level decomposition, Listing 6); with too few
 * sequences x heads to fill the chip the keys are split over several workgroups as well, whose
 * partial results are merged in a fixed order, by the one that comes last or by a second kernel. Weights are rounded
 * to `dtype` before they multiply V (Listing 5). The paper fixes no storage layout; this one is
 *   Q, O          device, contiguous [B, H, D]
 *   Kc, Vc        device, contiguous [num_blocks, H, block_size, D]: the cache, physical blocks
 *   block_table   device, int32 [B, max_blocks]: physical block of logical block i of sequence b;
 *                 logical key p is slot p % block_size of block block_table[b][p / block_size]
 *   seq_lens      device, int32 [B], 1 <= seq_lens[b] <= max_blocks * block_size
 * Table entries past the last used block are never read; cache slots are read in units of 16
 * keys, so the slots from seq_lens[b] up to the next multiple of 16 inside the last used block are
 * read and ignored (their weights are forced to zero), nothing beyond them. The library cannot inspect
 * device data: an entry outside [0, num_blocks) or a length outside its range is CLAMPED into it
 * (wrong result for that sequence, no out-of-range access).
 * D must be 64 or 128, block_size a multiple of 16 up to 1024 (else MLT_ERR_UNSUPPORTED); Q, Kc
 * and Vc 16-byte aligned, scale finite (MLT_ERR_INVALID_ARG). B or H equal to 0 is a no-op.
 */
int mlt_paged_attn_decode(int64_t B, int64_t H, int64_t D, int64_t block_size, int64_t max_blocks,
                          int64_t num_blocks, const void* Q, const void* Kc, const void* Vc,
                          const int32_t* block_table, const int32_t* seq_lens, void* O,
                          float scale, int dtype, void* stream);

/*
 * ---- 8 bits: weights and activations for mlt_gemm_fp8, and a paged cache of half the size.
 * e4m3 is the OCP format (1 sign, 4 exponent and 3 mantissa bits, largest value 448, NaN but no infinities), one byte an
 * element. A number is its e4m3 value times the fp32 scale of its block. The scales that the library writes are powers of
 * two: the smallest s >= 2^-100 with max |x| <= 448 s over the block's finite x, so that the rounding to e4m3 (to nearest, ties to
 * even) is the only one. Infinities and NaN become NaN. The scales that it reads may be any numbers from 2^-100 to 2^126,
 * and 0 for a block that counts as zeros.
 */

/*
 * Quantisation of a matrix to e4m3, with a scale for each block of 128 columns by block_rows rows: 1 (the rows of an activation)
 * or 128 (a weight).
 *   X       device, M x K row-major of `dtype`, row stride ldx >= K elements
 *   Xq      device, M x K row-major e4m3, row stride ldq >= K; written
 *   S       device, fp32 [ceil(K / 128)][ceil(M / block_rows)], row stride lds >= ceil(M / block_rows); written. The last
 *           block of a row or a column may be smaller.
 * K, ldx multiples of 8 and (with more than one row) ldq of 16, X and Xq 16-byte and S 4-byte aligned (else MLT_ERR_UNSUPPORTED for the sizes, MLT_ERR_INVALID_ARG for the
 * pointers); other block_rows: MLT_ERR_UNSUPPORTED. M or K equal to 0 is a no-op.
 */
int mlt_quant_fp8(int64_t M, int64_t K, const void* X, int64_t ldx, int64_t block_rows, void* Xq, int64_t ldq, float* S,
                  int64_t lds, int dtype, void* stream);

/*
 * The matrix product of e4m3 operands with block scales, C = A * B^T with B stored N x K:
 *   C[m][n] = sum over kb of Sa[kb][m] * Sb[kb][n / 128] * sum over k = 128 kb .. 128 kb + 127 of A[m][k] * B[n][k]
 * The matrix instruction adds the products of each aligned group of 8 k in fixed point: of every product it cuts off what lies
 * below 2^-13 of the largest one's power of two (that of A's number times that of B's). A group's sum is off by less than 7 * 2^-13 of its
 * largest |product|, which a sum that cancels can show: 448 * 448 - 448 * 448 + 1 * 1 in one group may give 0. The groups of a block are added
 * in fp32, a block's sum is multiplied by the product of its two scales (formed in fp32: beyond 2^128 it is infinite, below 2^-126 it loses bits), and the
 * sum over the blocks is fp32; C is rounded once to `dtype`. The order of the sums goes by the sizes and by B's alignment; equal calls
 * give equal bits.
 *   A       device, M x K row-major e4m3, row stride lda >= K
 *   Sa      device, fp32 [ceil(K / 128)][M], row stride ldsa >= M
 *   B       device, N x K row-major e4m3, row stride ldb >= K
 *   Sb      device, fp32 [ceil(K / 128)][ceil(N / 128)], row stride ldsb >= ceil(N / 128)
 *   C       device, M x N row-major of `dtype` (any alignment of its elements), row stride ldc >= N; written, never read
 * K, lda and ldb are multiples of 16 (MLT_ERR_UNSUPPORTED otherwise; fill up with zeros), A and B 16-byte, Sa, Sb 4-byte
 * aligned. M == 0 or N == 0 is a no-op, K == 0 stores zeros. Strides so large that 256 rows span 2^31 bytes:
 * MLT_ERR_UNSUPPORTED.
 */
int mlt_gemm_fp8(int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const float* Sa, int64_t ldsa, const void* B,
                 int64_t ldb, const float* Sb, int64_t ldsb, void* C, int64_t ldc, int dtype, void* stream);

/*
 * Appending to the cache of mlt_paged_attn_decode: the queries and keys of T new tokens are turned by the angles of their
 * positions, and the keys and values go to the slots that the block table names.
 *   Q, K, V      device, `dtype`: T rows of Hq, H and H heads of D elements side by side, row strides ldq, ldk, ldv (elements,
 *                multiples of 8: parts of one fused projection's result are fine). Hq may be 0 (no queries; Q, Qo unused).
 *   offsets      device, int32 [B + 1], 0 = offsets[0] <= offsets[1] <= ... <= T: rows offsets[b] .. offsets[b + 1] - 1 are
 *                the new tokens of sequence b, in order (none, one, many). Rows from offsets[B] on belong to nobody: they are
 *                not read, and nothing is written for them.
 *   seq_lens     device, int32 [B]: tokens of each sequence WITH the new ones, as the attention takes them afterwards. The
 *                i-th new token of sequence b has position seq_lens[b] - (offsets[b + 1] - offsets[b]) + i.
 *   block_table, Kc, Vc, block_size, max_blocks, num_blocks   as for mlt_paged_attn_decode, H the cache's heads
 *   cos, sin     device, fp32 [positions][rot / 2]. Of every head of Q and K the leading `rot` elements are turned, in pairs
 *                (x1, x2) -> (x1 cos - x2 sin, x2 cos + x1 sin) with the row of the token's position: elements i and i + rot / 2,
 *                or with `interleaved` != 0 elements 2 i and 2 i + 1. Computed in fp32, rounded once. rot = 0: none, cos
 *                and sin unused.
 *   Qo           device, contiguous [T, Hq, D]: the turned queries
 * A token whose position lies outside [0, max_blocks * block_size), or whose block number outside [0, num_blocks), is not written
 * to the cache; a position outside [0, positions) takes the nearest row of cos and sin. No two tokens may have one
 * slot. Slots of no new token keep what they hold. D must be 64 or 128, block_size a multiple of 16 up to 1024, rot a multiple of 16 up to D
 * (MLT_ERR_UNSUPPORTED); all tensors of `dtype` 16-byte aligned (MLT_ERR_INVALID_ARG). T or B equal to 0 is a no-op.
 */
int mlt_paged_append(int64_t T, int64_t B, int64_t Hq, int64_t H, int64_t D, int64_t block_size, int64_t max_blocks,
                     int64_t num_blocks, const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv,
                     const int32_t* offsets, const int32_t* seq_lens, const int32_t* block_table, const float* cos, const float* sin,
                     int64_t rot, int64_t positions, int interleaved, void* Qo, void* Kc, void* Vc, int dtype, void* stream);

/*
 * mlt_paged_append into an 8-bit cache:
 *   Kc, Vc       device, contiguous e4m3 [num_blocks, H, block_size, D]
 *   Ks, Vs       device, fp32 [num_blocks, H]: the scale of a block's keys (values) of one head
 * The turned keys are rounded from fp32 to e4m3. A block whose first slot is among the new ones starts afresh: its scale is
 * that of the new tokens. One that holds earlier tokens of its sequence keeps its scale (raised to a power of two) while it is large enough;
 * otherwise it takes the new tokens' scale, and the earlier tokens are rounded again in it. All new tokens of a
 * (block, head) are written by one owner: no two sequences may append to one block in one call. Otherwise as mlt_paged_append.
 */
int mlt_paged_append_fp8(int64_t T, int64_t B, int64_t Hq, int64_t H, int64_t D, int64_t block_size, int64_t max_blocks,
                         int64_t num_blocks, const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv,
                         const int32_t* offsets, const int32_t* seq_lens, const int32_t* block_table, const float* cos,
                         const float* sin, int64_t rot, int64_t positions, int interleaved, void* Qo, void* Kc, void* Vc, float* Ks,
                         float* Vs, int dtype, void* stream);

/*
 * mlt_paged_attn_decode over an 8-bit cache, with Hq / H query heads to each key/value head (query head q reads head
 * q / (Hq / H)):
 *   o = sum_j softmax_j(scale * q . k_j) v_j,   j = 0 .. seq_lens[b] - 1,   0 <= seq_lens[b] <= max_blocks * block_size
 *   Q, O          device, contiguous [B, Hq, D] of `dtype`
 *   Kc, Vc, Ks, Vs, block_table, block_size, max_blocks, num_blocks   as for mlt_paged_append_fp8
 * A sequence without keys gives zeros. The weights, each with the scale of its value, keep 22 bits whatever `dtype`, and whatever the other
 * keys' scales. Slots behind the last key are read in
 * units of 16 and ignored, as in mlt_paged_attn_decode, and so are the limits of what is read, the clamping of lengths (here
 * to 0 from below) and block numbers, and the requirements. H must divide Hq (MLT_ERR_INVALID_ARG).
 */
int mlt_paged_attn_decode_fp8(int64_t B, int64_t Hq, int64_t H, int64_t D, int64_t block_size, int64_t max_blocks,
                              int64_t num_blocks, const void* Q, const void* Kc, const void* Vc, const float* Ks, const float* Vs,
                              const int32_t* block_table, const int32_t* seq_lens, void* O, float scale, int dtype, void* stream);

/*
 * ---- Prompts, shared prefixes, 4-bit weights.
 */

/*
 * Attention forward of a batch of sequences of different lengths, packed one after the other, with Hq / H query heads to each key/value head
 * (query head q reads head q / (Hq / H)). For query i of the n of sequence b, over its m keys:
 *   o = sum_j softmax_j(scale * q . k_j) v_j,   j < m, with `causal` != 0 only j <= m - n + i
 * (the last query sees all keys: with n == m the lower triangle, with n < m the queries are the sequence's last tokens). A query that sees no key
 * (m == 0, or m < n) gives zeros.
 *   Q, K, V      device, `dtype`: Tq rows of Hq and Tk rows of H heads of D elements side by side, row strides ldq, ldk, ldv (elements, multiples of
 *                8: parts of one fused projection's result are fine)
 *   q_offsets    device, int32 [B + 1], 0 <= q_offsets[0] <= ... <= q_offsets[B] <= Tq: rows q_offsets[b] .. q_offsets[b + 1] - 1 of Q and O are
 *                sequence b's queries (none, one, many)
 *   k_offsets    device, int32 [B + 1], the same for its keys, up to Tk; may be q_offsets
 *   O            device, `dtype`: Tq rows of Hq heads, row stride ldo. Rows of no sequence are neither read nor written.
 * Weights are rounded to `dtype` before they multiply V, relative to a maximum of their row; their sum is that of the rounded ones (with the output's own rounding, outputs of random
 * inputs are off by 1.1 to 1.4 times what weights in fp32 would leave). What a query does not see
 * has no influence on it, whatever it holds (infinities and NaN too); one whose scores are all -inf gives zeros. Offsets out of their range or order give wrong results for their sequences, but no access out
 * of range. D must be 64 or 128, ldq, ldk, ldv, ldo multiples of 8, ldk and ldv below 2^23, ldo below 2^29, Tq, Tk, B, Hq * D and Tq * Hq / H below 2^29 (MLT_ERR_UNSUPPORTED); all tensors of `dtype`
 * 16-byte aligned, scale finite, H a divisor of Hq (MLT_ERR_INVALID_ARG). Tq, B or Hq equal to 0 is a no-op.
 */
int mlt_mha_packed_fwd(int64_t Tq, int64_t Tk, int64_t B, int64_t Hq, int64_t H, int64_t D, const void* Q, int64_t ldq, const void* K, int64_t ldk,
                       const void* V, int64_t ldv, const int32_t* q_offsets, const int32_t* k_offsets, void* O, int64_t ldo, float scale,
                       int causal, int dtype, void* stream);

/*
 * mlt_mha_packed_fwd with `causal`, for new tokens whose keys and values are in the paged cache already (mlt_paged_append puts them there):
 *   Q, ldq, O, ldo            as there, T rows
 *   offsets                   device, int32 [B + 1]: the rows of each sequence, as for mlt_paged_append
 *   seq_lens, block_table, Kc, Vc, block_size, max_blocks, num_blocks   as for mlt_paged_append: seq_lens[b] counts the sequence's tokens WITH the
 *                             new ones. The i-th of its n new tokens has position seq_lens[b] - n + i and sees the keys up to there.
 * A position below 0 gives zeros. Only slots below seq_lens[b] are read. Lengths are clamped to 0 .. max_blocks * block_size, block numbers to 0 .. num_blocks - 1 (wrong result
 * for that sequence, no access out of range). Requirements as for mlt_mha_packed_fwd; block_size a multiple of 16 up to 1024, max_blocks * block_size below 2^29.
 * The lengths are the device's, so it is the table's width, max_blocks * block_size, that decides whether few rows are spread over many workgroups: with a table far wider than the batch needs, a call
 * that is short by itself pays for that (33 tokens without history 8 us, with 32768 slots 13.5). A table cut to the batch's longest sequence avoids it.
 */
int mlt_paged_attn_prompt(int64_t T, int64_t B, int64_t Hq, int64_t H, int64_t D, int64_t block_size, int64_t max_blocks, int64_t num_blocks,
                          const void* Q, int64_t ldq, const void* Kc, const void* Vc, const int32_t* offsets, const int32_t* seq_lens,
                          const int32_t* block_table, void* O, int64_t ldo, float scale, int dtype, void* stream);

/*
 * mlt_paged_attn_decode for a batch whose sequences begin with the same prefix_len tokens, with Hq / H query heads to each key/value head. The prefix's
 * keys and values are read once for all sequences (by each of them where they are too few for that to pay):
 *   o = sum_j softmax_j(scale * q . k_j) v_j,   j = 0 .. seq_lens[b] - 1,   0 <= seq_lens[b] <= max_blocks * block_size
 *   Q, O           device, contiguous [B, Hq, D]
 *   Kc, Vc, block_size, max_blocks, num_blocks   as for mlt_paged_attn_decode
 *   prefix_table   device, int32 [ceil(prefix_len / block_size)]: the blocks of key 0 .. prefix_len - 1 (may be a row of block_table). prefix_len on the host; 0 for none
 *                  (prefix_table unused)
 *   block_table    device, int32 [B, max_blocks], as for mlt_paged_append: key j >= prefix_len of sequence b is in block block_table[b][j / block_size].
 *                  Entries below prefix_len / block_size are not read.
 *   seq_lens       device, int32 [B]: all of a sequence's tokens, the prefix's among them. A sequence may end inside the prefix; one without keys gives zeros.
 *   work           device, 16-byte aligned, work_bytes long: fp32 partial results, needed only while the call runs; or NULL: the library's scratch of the stream. With less than
 *                  mlt_paged_attn_decode_prefix_work says, or NULL on a stream that records into a graph, the prefix is read again for
 *                  every sequence. Two captured graphs that may run at the same time need a work of their own each.
 * How the work is spread goes by the table's width, as for mlt_paged_attn_prompt (64 sequences behind 8192 keys with 512 own ones 35 us, with 32768 slots a sequence 48).
 * Weights of own keys keep about 16 bits or more whatever `dtype`, as do those of the prefix where it is read for up to 32 queries of a key head (B * Hq / H) or by every sequence for itself; where it is read
 * once for more, they are rounded to `dtype`, as in mlt_mha_fwd. An infinity or NaN in a value makes the outputs of the sequences that see it non-finite. The limits of what is read, clamping and requirements are those of mlt_paged_attn_decode_fp8;
 * prefix_len must lie in 0 .. max_blocks * block_size (MLT_ERR_INVALID_ARG).
 */
int mlt_paged_attn_decode_prefix(int64_t B, int64_t Hq, int64_t H, int64_t D, int64_t block_size, int64_t max_blocks, int64_t num_blocks,
                                 const void* Q, const void* Kc, const void* Vc, const int32_t* prefix_table, int64_t prefix_len,
                                 const int32_t* block_table, const int32_t* seq_lens, void* O, float scale, void* work, int64_t work_bytes,
                                 int dtype, void* stream);

/* Bytes of `work` for a call of these sizes on the current device (0: the call needs none), or a negative mlt_status. */
int64_t mlt_paged_attn_decode_prefix_work(int64_t B, int64_t Hq, int64_t H, int64_t D, int64_t block_size, int64_t max_blocks, int64_t prefix_len);

/*
 * Few rows times a matrix of 4-bit weights: C = A * W^T, W[n][k] = S[k / group][n] * (q[n][k] - z),
 *   A       device, M x K row-major of `dtype`, row stride lda >= K
 *   Wq      device, N rows of K / 2 bytes, row stride ldw >= K / 2 bytes: q[n][k], 0 .. 15, is the low half of byte k / 2 of row n for even k, the high half for odd k
 *   S       device, `dtype` [ceil(K / group)][N], row stride lds >= N
 *   Z       device, uint8 [ceil(K / group)][N], row stride ldz >= N: z, 0 .. 15; or NULL: z = 8 (ldz unused)
 *   C       device, M x N row-major of `dtype`, row stride ldc >= N; written, never read
 * group is 32, 64 or 128; the last one of a row may be shorter. Products and the sum over a group are fp32, as is the sum over the groups, each times its scale; C is
 * rounded once. The sum over a group is taken as sum a (16 + q) less (16 + z) sum a: what fp32 loses goes by sum |a S| times up to 31 and not by |a (q - z) S|, some 2^-20 of a group's
 * sum |a S|. Where sums are not exact, a large element of A leaves that also at weights that equal their zero point. An infinity in a row of A, or a scale that is infinite, may give NaN in its row, or
 * column. The order of the sums goes by the sizes and by whether there is scratch to split K with (there is none where a stream records the call into a graph); equal calls give equal bits. K a multiple of 32, lda a multiple of 8,
 * ldw of 16, lda below 2^23, ldw below 2^24, lds and ldz below 2^26 (MLT_ERR_UNSUPPORTED); A and Wq 16-byte, S and C 2-byte aligned. M is taken up to 64 * 65535
 * (MLT_ERR_UNSUPPORTED; any with K == 0) as far as a launch has room for its tiles of 64 rows and 128 or 256 columns; the kernels are made for up to 64 rows (the weights are read again for every 64). M == 0 or N == 0 is a no-op, K == 0 stores zeros.
 */
int mlt_gemm_w4(int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const void* Wq, int64_t ldw, int64_t group, const void* S, int64_t lds,
                const uint8_t* Z, int64_t ldz, void* C, int64_t ldc, int dtype, void* stream);

/* Static, human-readable text for a status code. */
const char* mlt_status_string(int status);

/* Static version string, "major.minor.patch". */
const char* mlt_version(void);

#ifdef __cplusplus
}
#endif
#endif /* MLT_H_ */
