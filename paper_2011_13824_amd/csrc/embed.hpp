// Embedding: rows of a table by token, scaled, and the table's gradient.
//
//   out_i = scale * table[token_i]
//   dtable_v = base_v + scale * sum over {i : token_i = v} of dout_i
//
// A token outside [0, vocab) is padding: its row is 0, and it takes no part in the gradient.
//
// The gradient adds rows in the order of their positions, so the tokens are sorted first, stably.
// Up to kRankRows tokens every token counts those in front of it; more go through a radix sort.
// Both keep a few blocks busy, and the blocks behind them in the same launches write what no token
// names: zeros, or a copy of base.  The sorted tokens are then cut into pieces of equal length,
// whatever tokens they hold: a block sums the rows of each token of its piece and writes the sums
// of tokens that lie inside it, and those that cross an end go to the workspace and are joined in
// order by a second kernel.  So one token in all positions costs no more than all of them
// different, and no sum depends on the order in which blocks run.
#pragma once

#include "lm_types.hpp"

namespace lm {

template <typename T>
__global__ __launch_bounds__(256) void k_embed_fwd(const int64_t* __restrict__ tokens,
                                                   const T* __restrict__ table, int64_t ldt,
                                                   int64_t rows, int n, int vocab, float scale,
                                                   T* __restrict__ out, int64_t ldo) {
  const Piece p = piece_of((int64_t)blockIdx.x * 256, (n + 7) / 8);
  if (p.row >= rows) return;
  const int64_t t = load_global<int64_t>(tokens + p.row);
  const Columns<8> c(p.col, n);
  float v[8] = {};
  if (t >= 0 && t < vocab) {
    floats<T, 8>(load_columns<T, 8>(table + t * ldt, c), v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= scale;
  }
  store_columns<T, 8>(out + p.row * ldo, c, v);
}

// ---------------------------------------------------------------------------------------------
// The tokens in order
// ---------------------------------------------------------------------------------------------
struct Named {
  uint32_t token, at;  // padding has token vocab, behind all others
};
__device__ __forceinline__ Named load_named(const Named* p) {
  const u32x2 v = load_global<u32x2>(p);
  return Named{v[0], v[1]};
}

// Counting grows with the square: 4000 tokens 14 us in one launch, where the four launches of a
// radix sort take 16 to 20; 8000 would take some 45 us, the radix sort 18.
constexpr int kRankRows = 4096;
constexpr int kMaxDigit = 9;  // bits of a radix pass

// The part of a launch that fills the table's gradient: pieces [first, end) of 8 columns.  Rows
// that lie behind each other are one row (n = 0) of `values` values: a piece's place then takes no
// division, and odd widths no cut pieces (32003 rows of 1001 floats, copied: 45 us for 55).  Its
// stores pass the caches by, which the sums need: with 128000 x 4096 bf16 the fill takes 194 us for
// 175, and the sums behind it 34 for 68.
template <typename T>
struct EmbedFill {
  T* dtable;
  const T* base;  // NULL: zeros
  int64_t ldd, ldb, first, end, values;
  int n;
};

// A block fills kFillPieces pieces, a thread every 256th of them.
constexpr int kFillPieces = 256 * 8;

template <typename T>
__device__ __forceinline__ void embed_fill_flat(const EmbedFill<T>& f, int64_t block) {
  const int64_t p0 = f.first + block * kFillPieces + threadIdx.x;
  Vec<T, 8> v[kFillPieces / 256];
#pragma unroll
  for (int i = 0; i < kFillPieces / 256; ++i) {
    // behind the last whole piece the values before it again
    const int64_t at = min((p0 + i * 256) * 8, f.values - 8);
    if (f.base)
      v[i] = load_global<Vec<T, 8>>(f.base + at);
    else
      v[i] = Vec<T, 8>{};
  }
#pragma unroll
  for (int i = 0; i < kFillPieces / 256; ++i) {
    const int64_t at = min((p0 + i * 256) * 8, f.values - 8);
    if (p0 + i * 256 < f.end)
      __builtin_nontemporal_store(v[i],
                                  (__attribute__((address_space(1))) Vec<T, 8>*)(f.dtable + at));
  }
}

template <typename T>
__device__ __forceinline__ void embed_fill(const EmbedFill<T>& f, int64_t block) {
  if (f.n == 0) return embed_fill_flat(f, block);
  const int per_row = (f.n + 7) / 8;
  constexpr int kAhead = 4;
  for (int i0 = 0; i0 < kFillPieces / 256; i0 += kAhead) {
    Vec<T, 8> v[kAhead];
    if (f.base)
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int64_t start = f.first + block * kFillPieces + (i0 + i) * 256;
        if (start >= f.end) break;
        const Piece p = piece_of(start, per_row);
        // behind the end of the matrix the last row again
        const int64_t last = (f.end - 1) / per_row;
        v[i] = load_columns<T, 8>(f.base + min(p.row, last) * f.ldb, Columns<8>(p.col, f.n));
      }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int64_t start = f.first + block * kFillPieces + (i0 + i) * 256;
      if (start + threadIdx.x >= f.end) break;
      const Piece p = piece_of(start, per_row);
      float x[8] = {};
      if (f.base) floats<T, 8>(v[i], x);  // and back: exact
      store_columns<T, 8>(f.dtable + p.row * f.ldd, Columns<8>(p.col, f.n), x);
    }
  }
}

__device__ __forceinline__ uint32_t token_key(const int64_t* tokens, int64_t i, int vocab) {
  const int64_t t = load_global<int64_t>(tokens + i);
  return t >= 0 && t < vocab ? (uint32_t)t : (uint32_t)vocab;
}

// Up to kRankRows tokens: a block places 64, four threads each, a quarter of the comparisons a
// thread.  The blocks behind those fill.
template <typename T>
__global__ __launch_bounds__(256) void k_embed_rank(const int64_t* __restrict__ tokens, int rows,
                                                    int vocab, Named* __restrict__ out,
                                                    int sort_blocks, EmbedFill<T> fill) {
  if ((int)blockIdx.x >= sort_blocks) return embed_fill(fill, (int)blockIdx.x - sort_blocks);
  __shared__ __attribute__((aligned(16))) uint32_t keys[kRankRows];
  __shared__ int below[4][64];
  const int padded = (rows + 15) / 16 * 16;
  constexpr int kAhead = 8;
  for (int i0 = 0; i0 < padded; i0 += 256 * kAhead) {
    uint32_t key[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      key[j] = token_key(tokens, min(i0 + j * 256 + (int)threadIdx.x, rows - 1), vocab);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int i = i0 + j * 256 + threadIdx.x;
      if (i < padded) keys[i] = i < rows ? key[j] : 0xffffffffu;
    }
  }
  __syncthreads();
  const int lane = threadIdx.x & 63, part = threadIdx.x >> 6;
  const int first = blockIdx.x * 64, me = first + lane;
  const uint32_t key = me < rows ? keys[me] : 0u;
  const int from = part * (padded / 4), to = from + padded / 4;
  int count = 0;
  // in front of the block's own tokens equal ones count, behind them they do not
  auto take = [&](int i, int end, auto&& in_front) {
#pragma unroll 4
    for (; i < end; i += 4) {
      const u32x4 k = *(const u32x4*)(keys + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) count += in_front(k[j], i + j);
    }
  };
  take(from, min(to, first), [&](uint32_t k, int) { return k <= key; });
  take(max(from, first), min(to, first + 64),
       [&](uint32_t k, int i) { return k < key || (k == key && i < me); });
  take(max(from, first + 64), to, [&](uint32_t k, int) { return k < key; });
  below[part][lane] = count;
  __syncthreads();
  if (part == 0 && me < rows)
    out[below[0][lane] + below[1][lane] + below[2][lane] + below[3][lane]] =
        Named{key, (uint32_t)me};
}

// One radix pass, over `bits` bits from `shift` on: block b takes the `each` entries from b * each
// on, in `blocks` blocks.  The first pass reads the tokens (in = NULL).
struct RadixPass {
  const int64_t* tokens;
  const Named* in;
  Named* out;
  uint32_t* counts;  // [blocks][1 << bits]
  int64_t rows;
  int each, blocks, vocab, shift, bits;
};

__device__ __forceinline__ Named radix_entry(const RadixPass& r, int64_t i) {
  if (r.in) return load_named(r.in + i);
  return Named{token_key(r.tokens, i, r.vocab), (uint32_t)i};
}

// How many entries of a block have each digit.
template <typename T>
__global__ __launch_bounds__(256) void k_embed_count(RadixPass r, EmbedFill<T> fill) {
  if ((int)blockIdx.x >= r.blocks) return embed_fill(fill, (int)blockIdx.x - r.blocks);
  __shared__ uint32_t count[1 << kMaxDigit];
  const int bins = 1 << r.bits;
  for (int i = threadIdx.x; i < bins; i += 256) count[i] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * r.each, end = min(first + r.each, r.rows);
  for (int64_t i = first + threadIdx.x; i < end; i += 256)
    atomicAdd(&count[radix_entry(r, i).token >> r.shift & (bins - 1)], 1u);
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += 256) r.counts[(int64_t)blockIdx.x * bins + i] = count[i];
}

// Every entry to its place: behind all entries of lower digits, those of its digit in earlier
// blocks, and those in front of it in its block.
template <typename T>
__global__ __launch_bounds__(256) void k_embed_place(RadixPass r, EmbedFill<T> fill) {
  if ((int)blockIdx.x >= r.blocks) return embed_fill(fill, (int)blockIdx.x - r.blocks);
  __shared__ uint32_t next[1 << kMaxDigit], sum[256], mine[4][1 << kMaxDigit];
  const int bins = 1 << r.bits, t = threadIdx.x, lane = t & 63, wave = t >> 6;
  // digits 2t and 2t + 1: their entries in all blocks, and in the blocks before this one
  uint32_t all[2] = {}, before[2] = {};
  if (2 * t < bins) {
    for (int b = 0; b < r.blocks; ++b)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t c = 2 * t + j < bins ? r.counts[(int64_t)b * bins + 2 * t + j] : 0u;
        all[j] += c;
        if (b < (int)blockIdx.x) before[j] += c;
      }
  }
  sum[t] = all[0] + all[1];
  __syncthreads();
  for (int s = 1; s < 256; s <<= 1) {
    const uint32_t v = t >= s ? sum[t - s] : 0u;
    __syncthreads();
    sum[t] += v;
    __syncthreads();
  }
  const uint32_t lower = t ? sum[t - 1] : 0u;
  if (2 * t < bins) next[2 * t] = lower + before[0];
  if (2 * t + 1 < bins) next[2 * t + 1] = lower + all[0] + before[1];
  for (int i = t; i < 1 << kMaxDigit; i += 256) mine[0][i] = mine[1][i] = mine[2][i] = mine[3][i] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * r.each, end = min(first + r.each, r.rows);
  for (int64_t i0 = first; i0 < end; i0 += 256) {
    const int64_t i = i0 + t;
    const bool here = i < end;
    const Named e = here ? radix_entry(r, i) : Named{};
    const uint32_t digit = e.token >> r.shift & (bins - 1);
    uint64_t same = __ballot(here);  // lanes of the wave with this digit
    for (int b = 0; b < r.bits; ++b) {
      const uint64_t set = __ballot(digit >> b & 1);
      same &= digit >> b & 1 ? set : ~set;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
    if (here && rank == 0) mine[wave][digit] = __popcll(same);
    __syncthreads();
    uint32_t place = next[digit] + rank;
    for (int w = 0; w < wave; ++w) place += mine[w][digit];
    if (here) r.out[place] = e;
    __syncthreads();
    if (here && rank == 0) {  // each wave's count of a digit is added and cleared once
      atomicAdd(&next[digit], mine[wave][digit]);
      mine[wave][digit] = 0;
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------
// Sums of the rows of each token
// ---------------------------------------------------------------------------------------------
template <typename T>
struct EmbedSum {
  const Named* named;
  const T *dout, *base;
  T* dtable;
  float* part;  // [pieces][2][n]: the sum that a piece's first token ends with, or has over the
                // whole piece, where it began before; that which its last token begins with
  int64_t lddo, ldb, ldd, rows;
  int each, pieces, n, vocab;
  float scale;
};

template <typename T>
__device__ __forceinline__ void embed_write(const EmbedSum<T>& a, uint32_t token,
                                            const Columns<8>& c, const float (&sum)[8]) {
  float v[8] = {};
  if (a.base) floats<T, 8>(load_columns<T, 8>(a.base + token * a.ldb, c), v);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = fmaf(sum[i], a.scale, v[i]);
  store_columns<T, 8>(a.dtable + token * a.ldd, c, v);
}

// TX threads, 8 columns each, take a piece of a.each entries; 256 / TX pieces a block.  Eight rows
// are on their way at a time.
template <typename T, int TX>
__global__ __launch_bounds__(256) void k_embed_sum(EmbedSum<T> a, int slabs) {
  // a wave's threads have one piece: its tokens are the wave's, and so are the branches on them
  auto uniform = [](auto v) {
    return TX >= 64 ? (decltype(v))__builtin_amdgcn_readfirstlane((int)v) : v;
  };
  const int piece = uniform((int)(blockIdx.x / slabs) * (256 / TX) + (int)threadIdx.x / TX);
  const int col = (int)(blockIdx.x % slabs) * (TX * 8) + threadIdx.x % TX * 8;
  if (piece >= a.pieces || col >= a.n) return;
  const Columns<8> c(col, a.n);
  const int64_t first = (int64_t)piece * a.each, end = min(first + a.each, a.rows);
  constexpr int kAhead = 8;
  Named e[kAhead];
  auto names = [&](int64_t i0) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {  // past the end the last one again
      const Named v = load_named(a.named + min(i0 + j, end - 1));
      e[j] = Named{uniform(v.token), uniform(v.at)};
    }
  };
  const uint32_t before = uniform(load_named(a.named + max(first - 1, (int64_t)0)).token);
  uint32_t token = uniform(load_named(a.named + first).token);
  bool began = first == 0 || before != token;
  float sum[8] = {};
  for (int64_t i0 = first; i0 < end; i0 += kAhead) {
    Vec<T, 8> x[kAhead];
    names(i0);
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      x[j] = load_columns<T, 8>(a.dout + (int64_t)e[j].at * a.lddo, c);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (i0 + j >= end) break;
      if (e[j].token != token) {
        if (!began)
          store_columns<float, 8>(a.part + (int64_t)piece * 2 * a.n, c, sum);
        else if (token < (uint32_t)a.vocab)
          embed_write(a, token, c, sum);
        began = true;
        token = e[j].token;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) sum[k] += (float)x[j][k];
    }
  }
  const bool goes_on = end < a.rows && uniform(load_named(a.named + end).token) == token;
  if (!began || goes_on)
    store_columns<float, 8>(a.part + ((int64_t)piece * 2 + (began ? 1 : 0)) * a.n, c, sum);
  else if (token < (uint32_t)a.vocab)
    embed_write(a, token, c, sum);
}

// Joins a token that begins in `piece` and goes on behind it: 64 threads take 512 columns, four
// such groups every fourth of the pieces that follow, and the groups' sums are added in order.
template <typename T>
__global__ __launch_bounds__(256) void k_embed_join(EmbedSum<T> a, int slabs) {
  const int piece = (int)(blockIdx.x / slabs);
  const int64_t first = (int64_t)piece * a.each, end = first + a.each;
  const uint32_t token = load_named(a.named + end - 1).token;
  if (token >= (uint32_t)a.vocab) return;
  if (load_named(a.named + end).token != token) return;
  // a token that fills the piece and began before it is another piece's
  if (first > 0 && load_named(a.named + first - 1).token == token) return;
  // the last piece that holds the token: the first one whose next piece begins with another
  __shared__ int found;
  int last = piece + 1;
  for (;; last += 256) {
    if (threadIdx.x == 0) found = 256;
    __syncthreads();
    const int64_t next = ((int64_t)last + threadIdx.x + 1) * a.each;
    if (next >= a.rows || load_named(a.named + next).token != token)
      atomicMin(&found, (int)threadIdx.x);
    __syncthreads();
    const int f = found;
    __syncthreads();
    if (f < 256) {
      last += f;
      break;
    }
  }
  const int lane = threadIdx.x & 63, group = threadIdx.x >> 6;
  const int col = (int)(blockIdx.x % slabs) * 512 + lane * 8;
  const Columns<8> c(min(col, a.n - 1) / 8 * 8, a.n);
  __shared__ float all[3][64][8];
  float sum[8] = {};
  if (col < a.n) {
    if (group == 0)
      floats<float, 8>(load_columns<float, 8>(a.part + ((int64_t)piece * 2 + 1) * a.n, c), sum);
#pragma unroll 4
    for (int p = piece + 1 + group; p <= last; p += 4) {
      const Vec<float, 8> x = load_columns<float, 8>(a.part + (int64_t)p * 2 * a.n, c);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += x[i];
    }
  }
  if (group)
#pragma unroll
    for (int i = 0; i < 8; ++i) all[group - 1][lane][i] = sum[i];
  __syncthreads();
  if (group || col >= a.n) return;
#pragma unroll
  for (int g = 0; g < 3; ++g)
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] += all[g][lane][i];
  embed_write(a, token, c, sum);
}

}  // namespace lm
