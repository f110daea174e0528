// What the kernels of prompt.hip and prompt_ks.hip share: which item a workgroup takes, and where the rows of a sequence's queries, keys and values lie.
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

// The item of a workgroup: tile `tile` of the rows of one sequence and key/value head `h`; false: there is none left. The tiles of all sequences are taken in the order of
// their keys, most first, so that the launch ends with short ones: by the tokens that the tile's last row sees, in 64 steps of the longest sequence, within a step
// sequence by sequence. A sequence's tiles with at least L keys are its last (m - L) / tokens + 1 (a reciprocal's rounding moves a tile to the next step, the same
// way in every workgroup). `buf`: 6 * NT ints of LDS, free again afterwards (behind a barrier).
template <int ROWS, int NT>
__device__ __forceinline__ bool prompt_item(const PromptItems& a, int* buf, PromptSeq& seq, int& seq_b, int& h, int& tile) {
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
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  constexpr int NW = NT / 64;                            // (NW * 64 partial counts: NT ints)
  int *mm = buf, *tt = buf + NT, *part = buf + 2 * NT, *nn = buf + 3 * NT, *qq = buf + 4 * NT, *kk = buf + 5 * NT;
  auto tiles_of = [&](const PromptSeq& s) { return (int)(((int64_t)s.n * a.G + ROWS - 1) / ROWS); };
  // tiles of a sequence with at least L keys; L < 0: all of them
  auto at_least = [&](int m, int tiles, int L) {
    if (L < 0) return tiles;
    if (!a.causal) return m >= L ? tiles : 0;
    const float x = __builtin_floorf((float)(m - L) * a.r_tokens) + 1.f;
    return x <= 0.f ? 0 : x >= (float)tiles ? tiles : (int)x;
  };
  // the longest sequence
  int longest = 0;
  for (int b = tid; b < a.B; b += NT) {
    PromptSeq s;
    s.get(a, b);
    if (s.n > 0 && s.m > longest) longest = s.m;
    if (a.B <= NT) {                                     // all there are: kept
      mm[tid] = s.m;
      tt[tid] = tiles_of(s);
      nn[tid] = s.n;
      qq[tid] = s.q0;
      kk[tid] = s.k0;
    }
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
  for (int b0 = 0; b0 < a.B; b0 += NT) {
    if (a.B > NT) {                                      // these NT sequences
      PromptSeq s;
      s.m = 0; s.n = 0;
      if (b0 + tid < a.B) s.get(a, b0 + tid);
      __syncthreads();
      mm[tid] = s.m;
      tt[tid] = tiles_of(s);
      __syncthreads();
    }
    const int here = a.B - b0 < NT ? a.B - b0 : NT;
    for (int b = wave; b < here; b += NW) count += at_least(mm[b], tt[b], lane ? lane * step : -1);
  }
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
      int m = 0, tiles = 0;
      if (b0 + lane < a.B) {
        if (a.B <= NT) {
          m = mm[b0 + lane];
          tiles = tt[b0 + lane];
        } else {
          PromptSeq s;
          s.get(a, b0 + lane);
          m = s.m;
          tiles = tiles_of(s);
        }
      }
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
  if (found && a.B <= NT) {
    seq.q0 = uniform(qq[b]);
    seq.n = uniform(nn[b]);
    seq.k0 = uniform(kk[b]);
    seq.m = uniform(mm[b]);
  } else if (found) {
    seq.get(a, b);
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

// exponent all ones: a number that is not finite
template <typename Tag>
__device__ __forceinline__ bool wild(uint32_t pair, int half) {
  constexpr uint32_t E = __is_same(Tag, bf16_tag) ? 0x7f80u : 0x7c00u;
  return ((pair >> (16 * half)) & E) == E;
}

// By one wavefront, for rows q0 + r of its 32 whose outputs are not finite (bits r of `bad`): where a value that is not finite was among those that its tiles hold (up to key
// `held`; those from `there` on are key there - 1 again) and that the row does not see, the row is worked out again from the keys that it sees, one after the other
// (attn_rows.h), and stored. Returns the bits of those rows. (An accident of one token costs the rows around it that, and no others.)
template <typename Tag, int D, bool CAUSAL, bool PAGED>
__device__ __forceinline__ uint32_t prompt_redo(const PromptKernel& p, const PromptSeq& seq, int b, int head, int q0, uint32_t bad, int held, int there) {
  const int lane = threadIdx.x & 63, G = p.items.G, rows = seq.n * G;
  uint32_t redo = 0;
#pragma clang loop unroll(disable)
  while (bad) {
    const int r = __builtin_ctz(bad);
    bad &= bad - 1;
    if (q0 + r >= rows) break;
    const int tok = uniform((q0 + r) / G), g = q0 + r - tok * G, end = CAUSAL ? seq.m - seq.n + 1 + tok : seq.m;
    const int last = held < there ? held : there, first = held > there && end > there - 1 ? there - 1 : end;
    bool found = false;
#pragma clang loop unroll(disable)
    for (int key = (first > 0 ? first : 0) + lane; key < last; key += 64) {
      const uint16_t* v = prompt_value<D, PAGED>(p.src, seq, b, p.items.H, head, key);
#pragma clang loop unroll(disable)
      for (int d = 0; d < D; d += 2) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(v + d);
        found |= wild<Tag>(w, 0) || wild<Tag>(w, 1);
      }
    }
    if (!__any(found)) continue;
    redo |= 1u << r;
    const int64_t at = (int64_t)(head * G + g) * D;
    const uint16_t* q = p.Q + (int64_t)(seq.q0 + tok) * p.ldq + at;
    const float c = p.negate ? -p.c : p.c;
    attend_row<Tag, D>(q, p.O + (int64_t)(seq.q0 + tok) * p.ldo + at, end, [&](int64_t j) { return prompt_key<D, PAGED>(p.src, seq, b, p.items.H, head, (int)j); },
                       [&](int64_t j) { return prompt_value<D, PAGED>(p.src, seq, b, p.items.H, head, (int)j); }, c);
  }
  return redo;
}

}  // namespace mlt
