// What the kernels of prompt.hip, prompt_split.hip and (prompt_body) paged_prefix.hip share: which item a workgroup takes, and where the rows of a sequence's queries, keys and values lie.
//
// Rows. The G = Hq / H query heads that read one key/value head are rows of one matrix: row r of sequence b and key/value head h is query head h G + r % G
// of the sequence's token r / G. A tile of rows covers all of its tokens' heads, so that the keys are read once for all of them, and under the causal mask few tokens
// means that little of the diagonal is computed for nothing.
#pragma once

#include "attn_rows.h"
#include "mha_tile.h"

namespace mlt {

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }   // of a value that is one for the wavefront: in a scalar register

struct PromptItems {
  int T, Tk, B, H, G;
  const int32_t *q_offsets, *k_offsets, *seq_lens;   // seq_lens: lengths of the keys in a paged cache, instead of k_offsets
  int cap;                                           // ... and their limit
  int causal;
  int nxcd, teams, per_team, heads;                  // see PromptItem
  int tokens;                                        // whole tokens of a tile of rows (at least 1)
  float r_tokens;                                    // its reciprocal
};

// The host's part: XCDs in teams with `heads` key/value heads each (a divisor of both counts is the number of teams, so that each XCD's L2 holds as few heads'
// keys as can be), and workgroups for `rows`-row tiles of every sequence: no more than floor(T G / rows) + B for each head.
inline void prompt_teams(PromptItems& a, int64_t Hq, int64_t H, int rows, int nxcd) {
  a.H = (int)H;
  a.G = (int)(Hq / H);
  a.nxcd = nxcd;
  int g = nxcd, b = (int)H;
  while (b) { const int t = g % b; g = b; b = t; }
  a.teams = g;
  a.per_team = nxcd / g;
  a.heads = (int)H / g;
  a.tokens = rows / a.G > 0 ? rows / a.G : 1;
  a.r_tokens = 1.f / (float)a.tokens;
}
inline int64_t prompt_grid(const PromptItems& a, int rows) {
  const int64_t tiles = (int64_t)a.T * a.G / rows + a.B;
  return (tiles * a.heads + a.per_team - 1) / a.per_team * a.nxcd;
}

// Sequences up to which a workgroup finds its item in the order of the keys (prompt_item) and not in the batch's: it looks at all of them, in every workgroup. us sorted / in the batch's order, 32 heads
// over 8: 64 single tokens behind up to 4000 keys 97 / 127, 128 159 / 195, 256 355 / 385; but 128 ragged sequences of 16384 tokens 149 / 121, 256 195 / 124, 256 x 32 tokens 120 / 62, 512 x 16 312 / 109,
// 8192 single tokens 48500 / 1515. (8 to 32 sequences: the batch's order 2 to 17 % faster.)
constexpr int kPromptSorted = 128;

// rows q_offsets[b] .. of a sequence and its keys, with what is out of range put right
struct PromptSeq {
  int q0, n, k0, m;
  __device__ __forceinline__ void get(const PromptItems& a, int b) {
    auto in = [](int x, int hi) { return x < 0 ? 0 : x > hi ? hi : x; };
    q0 = in(a.q_offsets[b], a.T);
    n = in(a.q_offsets[b + 1], a.T) - q0;
    n = n < 0 ? 0 : n;
    if (a.seq_lens) {
      k0 = 0;
      m = in(a.seq_lens[b], a.cap);
    } else {
      k0 = in(a.k_offsets[b], a.Tk);
      m = in(a.k_offsets[b + 1], a.Tk) - k0;
      m = m < 0 ? 0 : m;
    }
  }
};

// Of more than kPromptSorted sequences: slot by slot in the batch's order. Sequence b has the slots from first(b) = floor(q0 G / ROWS) + b on, of which its tiles need no more than lie before first(b + 1)
// (floor(x + y) - floor(x) + 1 >= ceil(y)); the last b with first(b) <= slot is found by probes of 64 sequences at once, two rounds for 4096, whatever the offsets hold.
template <int ROWS>
__device__ __forceinline__ bool prompt_item_at(const PromptItems& a, int slot, PromptSeq& seq, int& seq_b, int& tile) {
  const int lane = threadIdx.x & 63;
  auto first = [&](int b) {
    const int q = a.q_offsets[b];
    return (int)((int64_t)(q < 0 ? 0 : q > a.T ? a.T : q) * a.G / ROWS) + b;
  };
  int lo = 0, n = a.B;
  while (n > 1) {
    const int step = (n + 63) / 64, at = lane * step;
    const unsigned long long in = __ballot(at < n && first(lo + (at < n ? at : 0)) <= slot);
    if (!in) return false;                                 // in front of the first sequence
    const int up = (63 - __builtin_clzll(in)) * step;
    lo += up;
    n = n - up < step ? n - up : step;
  }
  seq_b = lo;
  seq.get(a, lo);
  tile = (int)(((int64_t)seq.n * a.G + ROWS - 1) / ROWS) - 1 - (slot - first(lo));
  return tile >= 0;
}

// The item of a workgroup: tile `tile` of the rows of one sequence and key/value head `h`; false: there is none left. The tiles of all sequences are taken in the order of
// their keys, most first, so that the launch ends with short ones: by the tokens that the tile's last row sees, in 64 steps of the longest sequence, within a step
// sequence by sequence. A sequence's tiles with at least L keys are its last (m - L) / tokens + 1 (a reciprocal's rounding moves a tile to the next step, the same
// way in every workgroup). `buf`: 6 * NT ints of LDS, free again afterwards (behind a barrier).
template <int ROWS, int NT>
__device__ __forceinline__ bool prompt_item(const PromptItems& a, int* buf, PromptSeq& seq, int& seq_b, int& h, int& tile) {
  static_assert(kPromptSorted <= NT, "a thread for each sequence");
  const int xcd = (int)blockIdx.x % a.nxcd, idx = (int)blockIdx.x / a.nxcd * a.per_team + xcd / a.teams;
  h = xcd % a.teams * a.heads + idx % a.heads;
  int rank = idx / a.heads;
  if (a.B == 1) {
    seq_b = 0;
    seq.get(a, 0);
    const int tiles = (int)(((int64_t)seq.n * a.G + ROWS - 1) / ROWS);
    tile = tiles - 1 - rank;
    return tile >= 0;
  }
  if (a.B > kPromptSorted) return prompt_item_at<ROWS>(a, rank, seq, seq_b, tile);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  constexpr int NW = NT / 64;                            // (NW * 64 partial counts: NT ints)
  int *mm = buf, *tt = buf + NT, *part = buf + 2 * NT, *nn = buf + 3 * NT, *qq = buf + 4 * NT, *kk = buf + 5 * NT;
  // tiles of a sequence with at least L keys; L < 0: all of them
  auto at_least = [&](int m, int tiles, int L) {
    if (L < 0) return tiles;
    if (!a.causal) return m >= L ? tiles : 0;
    const float x = __builtin_floorf((float)(m - L) * a.r_tokens) + 1.f;
    return x <= 0.f ? 0 : x >= (float)tiles ? tiles : (int)x;
  };
  // the longest sequence
  int longest = 0;
  if (tid < a.B) {
    PromptSeq s;
    s.get(a, tid);
    if (s.n > 0) longest = s.m;
    mm[tid] = s.m;
    tt[tid] = (int)(((int64_t)s.n * a.G + ROWS - 1) / ROWS);
    nn[tid] = s.n;
    qq[tid] = s.q0;
    kk[tid] = s.k0;
  }
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) { const int o = __shfl_xor(longest, s); longest = o > longest ? o : longest; }
  if (lane == 0) part[wave] = longest;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) longest = part[w] > longest ? part[w] : longest;
  __syncthreads();
  const int step = longest / 64 + 1;
  // lane k: tiles with at least k * step keys (k = 0: all)
  int count = 0;
  for (int b = wave; b < a.B; b += NW) count += at_least(mm[b], tt[b], lane ? lane * step : -1);
  part[wave * 64 + lane] = count;
  __syncthreads();
  count = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) count += part[w * 64 + lane];
  // the last step that has more tiles than `rank` at or above it
  const unsigned long long more = __ballot(count > rank);
  const int k = more ? 63 - __builtin_clzll(more) : 0;
  bool found = more != 0;
  rank -= k < 63 ? __builtin_amdgcn_readlane(count, k + 1) : 0;
  const int lo = k ? k * step : -1, hi = k < 63 ? (k + 1) * step : 0x7fffffff;
  int b = 0;
  if (found) {
    found = false;
    for (int b0 = 0; b0 < a.B; b0 += 64) {               // every wavefront for itself
      const bool there = b0 + lane < a.B;
      const int m = there ? mm[b0 + lane] : 0, tiles = there ? tt[b0 + lane] : 0;
      const int above = at_least(m, tiles, hi), mine = at_least(m, tiles, lo) - above;
      int upto = mine;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) { const int o = __shfl_up(upto, d); upto += lane >= d ? o : 0; }
      const unsigned long long at = __ballot(upto > rank);
      if (at) {
        const int l = __builtin_ctzll(at);
        b = b0 + l;
        const int i = __builtin_amdgcn_readlane(above, l) + rank - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(mine, l));
        tile = __builtin_amdgcn_readlane(tiles, l) - 1 - i;
        found = true;
        break;
      }
      rank -= __builtin_amdgcn_readlane(upto, 63);
    }
  }
  b = __builtin_amdgcn_readfirstlane(b);
  if (found) {
    seq.q0 = uniform(qq[b]);
    seq.n = uniform(nn[b]);
    seq.k0 = uniform(kk[b]);
    seq.m = uniform(mm[b]);
  }
  seq_b = b;
  __syncthreads();
  return found && tile >= 0;
}

// Where a sequence's keys and values lie: packed rows, or blocks of a cache.
struct PromptKeys {
  const uint16_t *K, *V;
  int64_t ldk, ldv;                                  // packed
  const int32_t* block_table;                        // paged
  int block_size, max_blocks, num_blocks;
};

// An address that is one for the wavefront, in scalar registers (the direct loads take no other)
__device__ __forceinline__ const char* uniform(const char* p) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);
  return reinterpret_cast<const char*>((uint64_t)(uint32_t)uniform((int)(uint32_t)a) | (uint64_t)(uint32_t)uniform((int)(uint32_t)(a >> 32)) << 32);
}

// The way of one wavefront's loads through a sequence's keys (or values): N neighbouring ones that lie in one block of a cache (N divides 16), then those
// `step` further on. The block's number is read by the scalar unit when the ones before it are fetched. Keys past `last` (-1: there is none) are that one again.
template <int D, int N, bool PAGED>
struct PromptCursor {
  const char* base;
  int64_t row_bytes;                                 // packed: from a key to the next one; paged: D * 2
  const int32_t* table;
  int bs, last, last_blk, last_row, max_pb, per_block, step, step_blk, step_row;
  int key, blk, row, pb;                             // row: slot in the block
  __device__ __forceinline__ void start(const PromptKeys& src, const uint16_t* mat, int64_t ld, const PromptSeq& seq, int b, int heads, int h, int last_, int first, int step_) {
    last = last_;
    step = step_;
    key = first;
    blk = row = pb = 0;
    if constexpr (PAGED) {
      base = reinterpret_cast<const char*>(mat);
      row_bytes = D * 2;
      table = src.block_table + (int64_t)b * src.max_blocks;
      bs = src.block_size;
      max_pb = src.num_blocks - 1;
      per_block = heads * bs;
      step_blk = uniform(step / bs);
      step_row = step - step_blk * bs;
      blk = uniform(key / bs);
      last_blk = last >= 0 ? uniform(last / bs) : 0;
      last_row = last - last_blk * bs;
      row = key - blk * bs;
      base += (int64_t)h * bs * (D * 2);
      look_up();
    } else {
      base = reinterpret_cast<const char*>(mat + seq.k0 * ld + (int64_t)h * D);
      row_bytes = ld * 2;
    }
  }
  __device__ __forceinline__ void look_up() {
    // (through the constant address space: by the scalar unit. A vector load's wait would be one for the direct loads in flight too.)
    if (PAGED && last >= 0) pb = ((const __attribute__((address_space(4))) int32_t*)(uintptr_t)table)[key <= last ? blk : last_blk];
  }
  // the first of the N keys; `have`: how many of the others exist
  __device__ __forceinline__ const char* next(int& have) {
    const int over = key - last;                     // > 0: none of them exists
    have = over > 0 ? 0 : -over < N - 1 ? -over : N - 1;
    const char* p;
    if constexpr (PAGED) {
      const int blk_ok = pb < 0 ? 0 : pb > max_pb ? max_pb : pb;
      p = base + ((int64_t)blk_ok * per_block + (over > 0 ? last_row : row)) * (D * 2);
      blk += step_blk;
      row += step_row;
      if (row >= bs) { row -= bs; ++blk; }
    } else {
      p = base + (int64_t)(over > 0 ? last : key) * row_bytes;
    }
    key += step;
    look_up();
    return uniform(p);
  }
};

// Key (value) number `key` of a sequence (any below its count)
template <int D, bool PAGED>
__device__ __forceinline__ const uint16_t* prompt_row(const PromptKeys& src, const uint16_t* mat, int64_t ld, const PromptSeq& seq, int b, int H, int head, int key) {
  if constexpr (PAGED) {
    int pb = src.block_table[(int64_t)b * src.max_blocks + key / src.block_size];
    pb = pb < 0 ? 0 : pb >= src.num_blocks ? src.num_blocks - 1 : pb;
    return mat + (((int64_t)pb * H + head) * src.block_size + key % src.block_size) * D;
  } else {
    return mat + (int64_t)(seq.k0 + key) * ld + (int64_t)head * D;
  }
}
template <int D, bool PAGED>
__device__ __forceinline__ const uint16_t* prompt_key(const PromptKeys& src, const PromptSeq& seq, int b, int H, int head, int key) {
  return prompt_row<D, PAGED>(src, src.K, src.ldk, seq, b, H, head, key);
}
template <int D, bool PAGED>
__device__ __forceinline__ const uint16_t* prompt_value(const PromptKeys& src, const PromptSeq& seq, int b, int H, int head, int key) {
  return prompt_row<D, PAGED>(src, src.V, src.ldv, seq, b, H, head, key);
}

struct PromptKernel {
  const uint16_t* Q;
  uint16_t* O;
  PromptKeys src;
  PromptItems items;
  int64_t ldq, ldo;
  float c;
  int negate;
};

constexpr int kPromptPart = 512;                     // keys that a part of an item has at least

// prompt_split.hip: `parts` workgroups to an item; scratch: T * Hq * parts * (D + 2) numbers
int run_prompt_split(const PromptKernel& p, int dtype, int D, int64_t grid, int parts, float* scratch, hipStream_t s);

// What a number that is not finite is, in bits: 1 +inf, 2 -inf, 4 NaN; 0 for a finite one
template <typename Tag>
__device__ __forceinline__ uint32_t wild(uint16_t x) {
  constexpr uint32_t INF = __is_same(Tag, bf16_tag) ? 0x7f80u : 0x7c00u;
  const uint32_t a = x & 0x7fffu;
  return a < INF ? 0u : a > INF ? 4u : x >> 15 ? 2u : 1u;
}
// ... of values of both signs among what a sum has: NaN
__device__ __forceinline__ bool wild_nan(uint32_t w) { return w >= 3; }

// By one wavefront, after its rows have been stored: for rows q0 + r of its 32 whose outputs are not finite though the sums of their weights are (bits r of `bad`; of `none`: that sum is 0). The
// tiles hold keys up to `held`; those from `there` on are key there - 1 again. Where values that a row does not see are not finite, their weight of 0 has made NaN of the output's elements. Such an
// element is an infinity or NaN all the same if the row sees one there itself, which is found by looking at the values alone, one key after the other, once for all 32 rows (a row sees what
// the rows before it see). Otherwise the row is worked out again from the keys that it sees (attn_rows.h); these are rows in front of the first such value of an element, 64 tokens of each at most.
template <typename Tag, int D, bool CAUSAL, bool PAGED>
__device__ __forceinline__ void prompt_redo(const PromptKernel& p, const PromptSeq& seq, int b, int head, int q0, uint32_t bad, uint32_t none, int held, int there) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63, G = p.items.G, rows = seq.n * G;
  asm volatile("s_waitcnt vmcnt(0)" : : : "memory");       // what is stored here comes after what has been stored
  auto look = [&](int from, int to, uint32_t (&w)[E]) __attribute__((always_inline)) {   // elements 64 e + lane of values from .. to - 1
#pragma clang loop unroll(disable)
    for (int k0 = from; k0 < to; k0 += 8) {
      uint16_t x[8][E];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint16_t* v = prompt_value<D, PAGED>(p.src, seq, b, p.items.H, head, k0 + k < to ? k0 + k : to - 1);
#pragma unroll
        for (int e = 0; e < E; ++e) x[k][e] = v[64 * e + lane];
      }
#pragma unroll
      for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) w[e] |= wild<Tag>(x[k][e]);
      bool all = true;
#pragma unroll
      for (int e = 0; e < E; ++e) all = all && wild_nan(w[e]);
      if (__all(all)) break;                               // (it gets no worse)
    }
  };
  uint32_t seen[E] = {};
  int upto = 0;                                            // keys that `seen` has
#pragma clang loop unroll(disable)
  while (bad) {
    const int r = __builtin_ctz(bad);
    bad &= bad - 1;
    if (q0 + r >= rows) break;
    const int tok = uniform((q0 + r) / G), g = q0 + r - tok * G, end = CAUSAL ? seq.m - seq.n + 1 + tok : seq.m;
    const int last = held < there ? held : there, first = held > there && end > there - 1 ? there - 1 : end;
    uint32_t unseen[E] = {};
    look(first > 0 ? first : 0, last, unseen);
    bool some = false;
#pragma unroll
    for (int e = 0; e < E; ++e) some = some || unseen[e];
    if (!__any(some)) continue;
    if (end > upto) {
      look(upto, end, seen);
      upto = end;
    }
    bool again = none >> r & 1;
#pragma unroll
    for (int e = 0; e < E; ++e) again = again || (unseen[e] && !seen[e]);
    const int64_t at = (int64_t)(head * G + g) * D;
    uint16_t* out = p.O + (int64_t)(seq.q0 + tok) * p.ldo + at;
    if (__any(again)) {
      attend_row<Tag, D>(p.Q + (int64_t)(seq.q0 + tok) * p.ldq + at, out, end, [&](int64_t j) { return prompt_key<D, PAGED>(p.src, seq, b, p.items.H, head, (int)j); },
                         [&](int64_t j) { return prompt_value<D, PAGED>(p.src, seq, b, p.items.H, head, (int)j); }, p.negate ? -p.c : p.c);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (unseen[e]) out[64 * e + lane] = Elem<Tag>::from_f32(wild_nan(seen[e]) ? __builtin_nanf("") : seen[e] == 2 ? -__builtin_inff() : __builtin_inff());
    }
  }
}

// What a workgroup does of an item when its keys are split over several: tiles t0 .. t0 + tiles - 1 of them; the result goes, in fp32 and not divided by the sum, to
// o[(row * parts + part) * D ...], its maximum (log2 domain) and sum to s[(row * parts + part) * 2 ...]; row: of Q, all heads counted.
struct PromptPart {
  int t0, tiles, part, parts;
  float *o, *s;
};

// One item, by 8 wavefronts.
//
// The products, their schedule and the LDS ring are those of mha_pp.hip: workgroup = 8 wavefronts x 32 rows, key tiles of 64, S^T = K Q^T and O^T += V^T P^T on 32x32x16 MFMAs
// with P staying in registers, two groups of wavefronts half a tile apart (one in the softmax while the other one multiplies), tiles by direct loads into five slots.
// What differs:
//   * Rows are (token, head) pairs of a key/value head's whole group.
//   * A wavefront's loads of a tile are 8 neighbouring rows of K and of V. In a paged cache they lie in one block (blocks are whole multiples of 16 keys): one block
//     number for each tile, read by the scalar unit a tile ahead.
//   * A row may see no key at all: weights are taken against 0 while the maximum is -inf, and a sum of 0 gives an output of 0.
//   * A masked key's weight is 0, and 0 times a V that is not finite would be NaN. A row whose output is not finite, and to whose last tiles such a V belongs that it does not
//     see, is put right afterwards (prompt_redo). Nothing is spent on that before it is needed but one look at the outputs, 64 multiplications an item.
//
// 8192 tokens, 32 heads over 8, D = 128: 470 to 506 us on several cards, 1090 to 1170 TFLOP/s (the two-group kernel for a whole batch: 1150 to 1215); 512 tokens each of four sequences behind up to 8192 keys: 212 to 226 us. What bounds it is there the board's
// power and the exponentials beside the MFMAs, here that the longest of 272 items is as long as the call; with short sequences the start and end of an item, which nothing hides as a workgroup takes one item and a CU holds one
// workgroup (13 prompts of 8191 tokens in all: 89 to 92 us).
//
// The largest weight of a row lies between 1 and 2^8 (the reference moves when the maximum has grown by 8): fp16 weights lose nothing but what is below 2^-25 of it. Weights are
// rounded to 16 bits for the second product, and it is the rounded ones that are summed: what the rounding does to a row's weights as a whole cancels.
template <typename Tag, int D, bool CAUSAL, bool PAGED, bool SPLIT>
__device__ __forceinline__ void prompt_body(const PromptKernel& p, const PromptSeq& seq, int b, int head, int qt, uint32_t lds0, const PromptPart& part) {
  typedef PaCfg<D> L;
  typedef typename Elem<Tag>::vec8 V8;
  constexpr int NKK = L::NKK, NDT = L::NDT, ROWB = L::ROWB;
  constexpr int IN8 = 8 / L::LPW;                        // rows of one load
  const PromptKeys& src = p.src;
  const PromptItems& items = p.items;
  const int64_t ldq = p.ldq, ldo = p.ldo;
  const float c = p.c;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = wave >> 2;                             // waves w and w+4 share a SIMD
  const int lq = lane & 31, h = lane >> 5;
  const int G = items.G, rows = seq.n * G;
  const int key0 = SPLIT ? part.t0 * PA_BN : 0;          // keys are counted from here on
  const int m = SPLIT ? (seq.m - key0 < part.tiles * PA_BN ? seq.m - key0 : part.tiles * PA_BN) : seq.m;
  const int q0 = qt * PA_BM + wave * 32;                 // first row of this wavefront
  const int my_r = q0 + lq, last_r = rows - 1;
  const int my_tok = (my_r < last_r ? my_r : last_r) / G;   // (rows past the last one repeat it and are not stored)

  // Keys that row r sees: those before end(r) (all of them without the mask), none where that is 0 or less.
  const int shift = seq.m - key0 - seq.n + 1;
  auto end_of = [&](int r) {
    const int end = CAUSAL ? shift + uniform((r < last_r ? r : last_r) / G) : m;
    return SPLIT && end > m ? m : end;
  };
  const int wg_end = end_of((qt + 1) * PA_BM - 1), w_first = end_of(q0), w_end = end_of(q0 + 31), my_end = CAUSAL ? shift + my_tok : m;
  const int my_last = my_end - 1 - 4 * h;                // ... from the first key that this lane holds of 8
  const int nblk = wg_end > 0 ? (wg_end + PA_BN - 1) / PA_BN : 0;
  // This wavefront has visible keys in tiles 0 .. my_nblk-1 only.
  const int my_nblk = w_end > 0 && q0 < rows ? (w_end + PA_BN - 1) / PA_BN : 0;

  V8 qf[NKK];                                            // Q^T operand: row lq, d = 16*kk + 8*h .. +7

  // ---- global -> LDS assignments: wavefront w fills rows 8 w .. 8 w + 7 of the K tile and of the V tile; lane l owns the 16-byte slot l of a 1 KB block.
  const uint32_t rowk = PAGED ? ROWB : (uint32_t)src.ldk * 2, rowv = PAGED ? ROWB : (uint32_t)src.ldv * 2;
  uint32_t voff_k[L::LPW], voff_v[L::LPW];               // byte offsets from the first of the 8 rows, all of them there
  // `have`: rows behind the first one that are there; those past them re-read the last one (their weights are 0)
  auto offsets_of = [&](int ln, int i, int have, uint32_t& ok, uint32_t& ov) __attribute__((always_inline)) {
    const int in8 = i * IN8 + ln / L::CPR, slot = ln % L::CPR, at = in8 < have ? in8 : have;
    ok = (uint32_t)at * rowk + (uint32_t)(slot ^ L::fk(wave * 8 + in8)) * 16u;
    ov = (uint32_t)at * rowv + (uint32_t)(slot ^ L::fv(wave * 8 + in8)) * 16u;
  };
#pragma unroll
  for (int i = 0; i < L::LPW; ++i) offsets_of(lane, i, 7, voff_k[i], voff_v[i]);
  const int last_key = key0 + wg_end - 1;                // of what this workgroup reads
  PromptCursor<D, 8, PAGED> at;                          // (K and V of a packed sequence may have other strides: ...)
  auto first_tile = [&]() __attribute__((always_inline)) { at.start(src, src.K, src.ldk, seq, b, items.H, head, wg_end > 0 ? last_key : -1, key0 + wave * 8, PA_BN); };
  auto issue_tile = [&](int t) __attribute__((always_inline)) {
    const uint32_t dst = lds0 + (t % PA_NS) * L::SLOT_B + wave * L::LPW * 1024;
    int have;
    const int key = at.key < last_key ? at.key : last_key;
    const char* kp = at.next(have);
    const char* vp = uniform(PAGED ? reinterpret_cast<const char*>(src.V) + (kp - reinterpret_cast<const char*>(src.K))
                                   : reinterpret_cast<const char*>(src.V + (int64_t)(seq.k0 + key) * src.ldv + (int64_t)head * D));   // (... this is V's)
    if (D == 128 && have == 7) {                         // (D = 64 has no registers to keep them in)
#pragma unroll
      for (int i = 0; i < L::LPW; ++i) load_lds16(kp, voff_k[i], dst + i * 1024);
#pragma unroll
      for (int i = 0; i < L::LPW; ++i) load_lds16(vp, voff_v[i], dst + L::TILE_B + i * 1024);
    } else {
      int ln = lane;
      asm volatile("" : "+v"(ln));
#pragma unroll
      for (int i = 0; i < L::LPW; ++i) {
        uint32_t ok, ov;
        offsets_of(ln, i, have, ok, ov);
        load_lds16(kp, ok, dst + i * 1024);
        load_lds16(vp, ov, dst + L::TILE_B + i * 1024);
      }
    }
  };

  f32x16 o_acc[NDT];
  f32x16 s_acc[2];
  u32x4 pq[4];                       // P^T of the current tile as MFMA operands: one per 16 keys
  float mc_run, l_run;
  V8 fb[2][NDT];
  // Fragment addresses: one per XOR variant in a register, moved from slot to slot; D = 64, which has no registers to spare, keeps one of K's and works out the others
  constexpr int NKA = D == 64 ? 1 : NKK;
  uint32_t ka[NKA], va[NDT];
  auto read_v_frag = [&](int g, int t, V8& f) {
    const uint32_t a = va[t] + g * 16 * ROWB;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((MLT_LDS s16x4*)(uintptr_t)a);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((MLT_LDS s16x4*)(uintptr_t)(a + 8 * ROWB));
    f = join_tr<V8>(lo, hi);
  };
  auto read_k_frag = [&](int fi, V8& f) {
    const uint32_t a = (NKA == 1 ? ka[0] ^ ((fi >> 1) << 5) : ka[(fi >> 1) % NKA]) + (fi & 1) * 32 * ROWB;
    f = __builtin_bit_cast(V8, *(const MLT_LDS u32x4*)(uintptr_t)a);
  };
  auto mfma_v = [&](int g, int t, const V8& f) { o_acc[t] = mfma32(f, __builtin_bit_cast(V8, pq[g]), o_acc[t]); };
  auto mfma_k = [&](int fi, const V8& f) {
    if (fi < 2) {
      f32x16 z;
#pragma unroll
      for (int r = 0; r < 16; ++r) z[r] = 0.f;
      s_acc[fi & 1] = mfma32(f, qf[fi >> 1], z);
    } else {
      s_acc[fi & 1] = mfma32(f, qf[fi >> 1], s_acc[fi & 1]);
    }
  };
#define MLT_SB() __builtin_amdgcn_sched_barrier(0)
  auto cut = [&](int j) { return (j + 1) * PA_BN > w_first; };         // does the mask, or the last key, cut tile j for this wavefront?

  // ---- softmax of S_j (in s_acc) -> pq, mc_run, rescaled o_acc and l_run (see mha_pp_kernel)
  auto softmax_tile = [&](int j) {
    // register r of sub-tile kb is key 64 j + 32 kb + 8 (r / 4) + 4 h + r % 4
    if (cut(j)) {
      const int rel = my_last - j * PA_BN;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * kb + 8 * (r >> 2) + (r & 3) > rel) s_acc[kb][r] = -__builtin_inff();
    }
    float mx = max3(s_acc[0][0], s_acc[0][1], s_acc[0][2]);
#pragma unroll
    for (int r = 3; r < 15; r += 2) mx = max3(mx, s_acc[0][r], s_acc[0][r + 1]);
    mx = max3(mx, s_acc[0][15], s_acc[1][0]);
#pragma unroll
    for (int r = 1; r < 15; r += 2) mx = max3(mx, s_acc[1][r], s_acc[1][r + 1]);
    mx = __builtin_fmaxf(mx, s_acc[1][15]);
    mx = both_halves_max(mx);
    const float t = mx * c;
    const bool grow = t - mc_run > PA_LAZY_T;
    if (__builtin_amdgcn_ballot_w64(grow) != 0) {
      const float alpha = grow ? __builtin_amdgcn_exp2f(mc_run - t) : 1.f;
      l_run *= alpha;
#pragma unroll
      for (int tt = 0; tt < NDT; ++tt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o_acc[tt][r] *= alpha;
      mc_run = grow ? t : mc_run;
    }
    const float ref = mc_run == -__builtin_inff() ? 0.f : mc_run;        // (no key seen yet: all weights are exp2(-inf))
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s_acc[kb][r], c, -ref));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s_acc[kb][r + 1], c, -ref));
        pq[2 * kb + r / 8][(r / 2) & 3] = Elem<Tag>::pack2(p0, p1);
      }
  };
  constexpr int LPT = 2 * L::LPW;                         // loads per wavefront per tile
#pragma unroll
  for (int t = 0; t < NDT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) o_acc[t][r] = 0.f;
  mc_run = -__builtin_inff();    // reference point of the weights: a running maximum of the scores, times c (log2 domain)
  l_run = 0.f;                   // running sum over this lane's half of the keys
  {
    // Q, and fragment addresses inside a slot (see mha_pp_kernel), from an opaque lane number: not to be kept in registers for a second turn
    int ln = lane;
    asm volatile("" : "+v"(ln));
    const int fq = ln & 31, fh = ln >> 5;
    const int row = q0 + fq < last_r ? q0 + fq : last_r, tok = row / G;
    const uint16_t* qp = p.Q + (int64_t)(seq.q0 + tok) * ldq + (int64_t)(head * G + row - tok * G) * D + 8 * fh;
    const uint32_t flip = p.negate ? 0x80008000u : 0u;       // a negative scale as a sign flip
#pragma unroll
    for (int kk = 0; kk < NKK; ++kk) {
      u32x4 raw = *reinterpret_cast<const u32x4_mem*>(qp + kk * 16);
      raw[0] ^= flip; raw[1] ^= flip; raw[2] ^= flip; raw[3] ^= flip;
      qf[kk] = __builtin_bit_cast(V8, raw);
    }
    const int k_frag = fq * ROWB + ((fh ^ L::fk(fq)) << 4);
    const int vg = ln >> 4, vs = ln & 15;
    const int v_row = 4 * (vg >> 1) + (vs >> 2);
    const int v_frag = L::TILE_B + v_row * ROWB + (((2 * (vg & 1) + ((vs & 3) >> 1)) ^ L::fv(v_row)) << 4) + 8 * (vs & 1);
#pragma unroll
    for (int kk = 0; kk < NKA; ++kk) ka[kk] = lds0 + (uint32_t)(k_frag ^ (kk << 5));
#pragma unroll
    for (int t = 0; t < NDT; ++t) va[t] = lds0 + (uint32_t)(v_frag ^ (t << 6));
  }

  // ---- schedule: see mha_pp_kernel
  first_tile();
#pragma unroll
  for (int t = 0; t < PA_AHEAD; ++t)
    if (t < nblk) issue_tile(t);
  if (nblk >= 3) __builtin_amdgcn_s_waitcnt(wait_imm(2 * LPT, 15));
  else if (nblk == 2) __builtin_amdgcn_s_waitcnt(wait_imm(LPT, 15));
  else __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));
  MLT_BARRIER();
  if (grp == 1) MLT_BARRIER();            // stagger: group 1 runs one phase behind
  {
    if (my_nblk > 0) {                                    // ka, va point into slot 0
#pragma unroll
      for (int i = 0; i < NDT; ++i) read_k_frag(i, fb[0][i]);
#pragma unroll
      for (int i = 0; i < NDT; ++i) read_k_frag(NDT + i, fb[1][i]);
      MLT_SB();
#pragma unroll
      for (int ch = 0; ch < 4; ++ch)
#pragma unroll
        for (int i = 0; i < NDT; ++i) {
          mfma_k(ch * NDT + i, fb[ch & 1][i]);
          MLT_SB();
          if (ch < 2) read_k_frag((ch + 2) * NDT + i, fb[ch & 1][i]);
          else read_v_frag(ch - 2, i, fb[ch & 1][i]);
          MLT_SB();
        }
    }
    if (grp == 1) {
      if (nblk >= 3) __builtin_amdgcn_s_waitcnt(wait_imm(LPT, 15));
      else __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));
    }
    MLT_BARRIER();
  }

  int slot_off = 0;                                       // byte offset of tile j's slot
  for (int j = 0; j < nblk; ++j) {
    const int slot_off_next = slot_off + L::SLOT_B == L::SMEM ? 0 : slot_off + L::SLOT_B;
    const bool active = j < my_nblk;                       // wavefront-uniform
    const bool active_next = j + 1 < my_nblk;
    // ---- X_j (the first two V_j groups are already in the chunk buffers)
    if (j + PA_AHEAD < nblk) issue_tile(j + PA_AHEAD);
    __builtin_amdgcn_sched_barrier(0);
    if (active) {
      softmax_tile(j);
#pragma unroll
      for (int g = 0; g < 4; ++g) asm volatile("" : "+v"(pq[g]));
    }
    __builtin_amdgcn_sched_barrier(0);
    if (grp == 0) {
      const int newer = (j + 3 < nblk ? 1 : 0) + (j + 2 < nblk ? 1 : 0);
      if (newer == 2) __builtin_amdgcn_s_waitcnt(wait_imm(2 * LPT, 0));
      else if (newer == 1) __builtin_amdgcn_s_waitcnt(wait_imm(LPT, 0));
      else __builtin_amdgcn_s_waitcnt(wait_imm(0, 0));
    } else {
      __builtin_amdgcn_s_waitcnt(wait_imm(63, 0));
    }
    MLT_BARRIER();
    __builtin_amdgcn_sched_barrier(0);
    if (D == 128) __builtin_amdgcn_s_setprio(1);
    // ---- C_j
    if (active) {
      const uint32_t dslot = (uint32_t)(slot_off_next - slot_off);
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int t = 0; t < NDT; ++t) {
          mfma_v(g, t, fb[g & 1][t]);
          MLT_SB();
          if (g < 2) read_v_frag(g + 2, t, fb[g & 1][t]);
          else read_k_frag((g - 2) * NDT + t, fb[g & 1][t]);
          if (g == 0 && NKA > 1) { ka[(2 * t) % NKA] += dslot; ka[(2 * t + 1) % NKA] += dslot; }
          if (g == 0 && NKA == 1 && t == 0) ka[0] += dslot;
          if (g == 3) va[t] += dslot;
          MLT_SB();
        }
      if (active_next) {
#pragma unroll
        for (int ch = 0; ch < 4; ++ch)
#pragma unroll
          for (int i = 0; i < NDT; ++i) {
            mfma_k(ch * NDT + i, fb[ch & 1][i]);
            MLT_SB();
            if (ch < 2) read_k_frag((ch + 2) * NDT + i, fb[ch & 1][i]);
            else read_v_frag(ch - 2, i, fb[ch & 1][i]);
            MLT_SB();
          }
      }
      // the sum of the ROUNDED weights (what P V used), while the matrix pipe drains
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) l_run = Elem<Tag>::add_pair(pq[g][e], l_run);
      asm volatile("" : "+v"(l_run));
    }
    if (D == 128) __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
    if (grp == 1) {
      if (j + 3 < nblk) __builtin_amdgcn_s_waitcnt(wait_imm(LPT, 15));
      else __builtin_amdgcn_s_waitcnt(wait_imm(0, 15));
    }
    MLT_BARRIER();
    __builtin_amdgcn_sched_barrier(0);
    slot_off = slot_off_next;
  }
  if (grp == 0) MLT_BARRIER();            // same barrier count for both groups

#undef MLT_SB
  const float l_tot = both_halves_sum(l_run);
  if constexpr (SPLIT) {
    if (my_r < rows) {
      const int64_t at = ((int64_t)(seq.q0 + my_tok) * (items.H * G) + head * G + (my_r - my_tok * G)) * part.parts + part.part;
      if (h == 0) {
        part.s[2 * at] = mc_run;
        part.s[2 * at + 1] = l_tot;
      }
      if (nblk == 0) return;                             // (no keys: nothing that anyone reads)
      // register quad g of tile t holds d = 32 t + 8 g + 4 h .. + 3
#pragma unroll
      for (int t = 0; t < NDT; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<f32x4_mem*>(part.o + at * D + 32 * t + 8 * g + 4 * h) = f32x4{o_acc[t][4 * g], o_acc[t][4 * g + 1], o_acc[t][4 * g + 2], o_acc[t][4 * g + 3]};
    }
    return;
  }

  // ---- rows to be looked at again (prompt_redo): an output is not finite, though the sum of the weights is
  float sum = 0.f;                          // x * 0 is 0, or NaN where x is not finite
#pragma unroll
  for (int t = 0; t < NDT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) sum = __builtin_fmaf(o_acc[t][r], 0.f, sum);
  const uint64_t bad = __builtin_amdgcn_ballot_w64(!(sum == 0.f) && l_tot - l_tot == 0.f), none = __builtin_amdgcn_ballot_w64(l_tot == 0.f);

  // ---- epilogue: O = O^T / l, l summed over both key halves, rows without keys 0; whole rows through LDS, 16 bytes a lane
  const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
  u32x4 ow[NDT][2];
#pragma unroll
  for (int t = 0; t < NDT; ++t)
#pragma unroll
    for (int gp = 0; gp < 2; ++gp) ow[t][gp] = o_piece16<Tag>(o_acc[t], 2 * gp, inv);
  const uint32_t o_lds = lds0 + wave * 32 * ROWB;
  constexpr int CM = L::CPR - 1;
#pragma unroll
  for (int t = 0; t < NDT; ++t)
#pragma unroll
    for (int gp = 0; gp < 2; ++gp) {
      const int ch = 4 * t + 2 * gp + h;
      *(MLT_LDS u32x4*)(uintptr_t)(o_lds + lq * ROWB + ((ch ^ (lq & CM)) << 4)) = ow[t][gp];
    }
  // where row lq goes, in 16-byte pieces from the wavefront's first token on (a store writes whole rows and asks the lane that knows). Worked out again rather than kept in
  // registers through the loop.
  int ln = lane;
  asm volatile("" : "+v"(ln));
  const int out_row = q0 + (ln & 31) < last_r ? q0 + (ln & 31) : last_r, out_tok = out_row / G, tok0 = uniform((q0 < last_r ? q0 : last_r) / G);
  const int o_piece = (int)(((out_tok - tok0) * ldo + (int64_t)(out_row - out_tok * G) * D) / 8);
  uint16_t* ob = p.O + (int64_t)(seq.q0 + tok0) * ldo + (int64_t)head * G * D;
#pragma unroll
  for (int i = 0; i < 32 / L::RPB; ++i) {
    const int r = i * L::RPB + lane / L::CPR, cc = lane % L::CPR;
    const u32x4 v = *(const MLT_LDS u32x4*)(uintptr_t)(o_lds + r * ROWB + ((cc ^ (r & CM)) << 4));
    const int piece = __shfl(o_piece, r);
    if (q0 + r < rows) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_mem*>(ob + ((int64_t)piece + cc) * 8));
  }
  if (bad) prompt_redo<Tag, D, CAUSAL, PAGED>(p, seq, b, head, q0, (uint32_t)bad | (uint32_t)(bad >> 32), (uint32_t)none, my_nblk * PA_BN, wg_end);
}

}  // namespace mlt
