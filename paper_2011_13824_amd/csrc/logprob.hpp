// Log probabilities of given tokens, entropy and the most likely tokens of rows of logits, and the
// gradient of the first two.
//
//   d_j = scale (l_j - max l),  S = sum e^d,  lse = scale max l + log S
//   logp = d_token - log S,     H = log S - (sum e^d d) / S
//   dl_j = scale (g ([j = token] - p_j) - h p_j (log p_j + H)),  p_j = e^(scale l_j - lse)
//
// A row is read once: a thread keeps the largest logit that it has met and both sums relative to
// it, and scales the sums where a larger one comes.  Differences to the maximum are taken before
// they are scaled, so no magnitude of the logits costs the probabilities accuracy.
//
// The most likely tokens: a thread also keeps which eight columns held its largest logit.  Among
// the threads' best, ordered by value and then by column, the top-th bounds the answer from below,
// so the `top` threads at or above it hold all of it; they read their columns again, and what
// reaches the bound (a few more than `top`, at most all that these threads have) is put in order by
// counting. Equal logits, all equal ones too, change neither the result's order nor the bound on
// the work.
//
// Few rows are split over blocks of at least kPartColumns columns; a second launch joins the parts
// in the same way.
//
// Bound by bytes and nearly as much by the vector units (9 instructions and an exponential of two a
// logit).  4096 rows of 128000 bf16 logits: 187 us for 1.05 GB (5.6 TB/s, vector units 87 % busy),
// the gradient 405 us for 2.1 GB (5.2 TB/s, 68 %).  With alternatives, of which each row's block
// makes its own search, those 4096 rows take 213 us for 5, 259 for 20 and 300 for 32 where they take
// 202 without (other logits than above).  One row of 128000 with 20 alternatives: 10 + 8 us, latency.
#pragma once

#include "lm_types.hpp"

namespace lm {

constexpr int kTop = 32;              // most likely tokens that a call may ask for
constexpr int kMaxParts = 256;
constexpr int kPartColumns = 256 * 8;
constexpr int kBackColumns = 256 * 8 * 4;  // of a block of the gradient
constexpr float kFar = -200.f;  // e^kFar is 0 in 32 bits; a product with it is finite

// Values in the order of the numbers, equal values from the lowest column on: a larger key comes
// first.  -0 and 0 are equal.  0 stands for none.
__device__ __forceinline__ uint64_t rank_key(float v, uint32_t column) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return (uint64_t)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | ~column;
}
__device__ __forceinline__ float key_value(uint64_t key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint32_t key_column(uint64_t key) { return ~(uint32_t)key; }

// The largest logit, and the sums of e^d and e^d d relative to it.  Without a logit over -inf
// `most` is the lowest float and both sums are 0; a NaN stays in `most` for good.
struct Sums {
  float most, total, moment;
};
__device__ __forceinline__ Sums no_sums() { return Sums{-3.402823466e+38f, 0.f, 0.f}; }

__device__ __forceinline__ void rescale(Sums& s, float most, float scale) {
  const float d = __builtin_elementwise_maximum((s.most - most) * scale, kFar);
  const float c = __expf(d);
  s.moment = c * fmaf(s.total, d, s.moment);
  s.total *= c;
  s.most = most;
}
__device__ __forceinline__ Sums joined(Sums a, Sums b, float scale) {
  const float most = __builtin_elementwise_maximum(a.most, b.most);
  rescale(a, most, scale);
  rescale(b, most, scale);
  return Sums{most, a.total + b.total, a.moment + b.moment};
}

template <typename T>
struct LogProb {
  const T* logits;
  int64_t ldl, rows;
  int n, parts, part_columns, top;
  float scale;
  const int64_t* tokens;
  float *logp, *lse, *entropy, *top_logp;
  int64_t* top_tokens;
  Sums* part_sums;      // [rows][parts]
  uint64_t* part_keys;  // [rows][parts][top], largest first, 0 behind the last
};

// Adds eight logits, `most` the largest of them, to sums in powers of two (to2 = scale / log 2): the
// moment is log 2 times too small.
__device__ __forceinline__ void add8(Sums& s, const float (&x)[8], float most, float to2) {
  if (!(most <= s.most)) {  // a NaN too
    const float d = __builtin_elementwise_maximum((s.most - most) * to2, kFar);
    const float c = __builtin_amdgcn_exp2f(d);
    s.moment = c * fmaf(s.total, d, s.moment);
    s.total *= c;
    s.most = __builtin_elementwise_maximum(s.most, most);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float d = __builtin_elementwise_maximum((x[i] - s.most) * to2, kFar);
    const float e = __builtin_amdgcn_exp2f(d);
    s.total += e;
    s.moment = fmaf(e, d, s.moment);
  }
}
__device__ __forceinline__ float largest(const float (&x)[8]) {
  float most = x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) most = __builtin_elementwise_maximum(most, x[i]);
  return most;
}

// Calls f(eight logits, their first column) for the columns [first, end) of a row: a thread takes
// every 256th eight, the last of them with -inf behind the end.
constexpr int kStep = 256 * 8;
template <typename T, typename F>
__device__ __forceinline__ void walk(const T* l, int first, int end, F&& f) {
  constexpr int kAhead = 4;
  int col = first + threadIdx.x * 8;
  for (; col + (kAhead - 1) * kStep + 8 <= end; col += kAhead * kStep) {
    Vec<T, 8> x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) x[u] = load_global<Vec<T, 8>>(l + col + u * kStep);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (float)x[u][i];
      f(v, col + u * kStep);
    }
  }
  for (; col < end; col += kStep) {
    float v[8];
    load_row_end<T, 8>(l + col, end - col, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < end - col ? v[i] : -__builtin_inff();
    f(v, col);
  }
}

// Sums of 256 threads in one order; thread 0 has the result.
__device__ __forceinline__ Sums block_sums(Sums s, float scale, Sums* shared) {
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    Sums o;
    o.most = __shfl_xor(s.most, d);
    o.total = __shfl_xor(s.total, d);
    o.moment = __shfl_xor(s.moment, d);
    s = joined(s, o, scale);
  }
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0)
    for (int w = 1; w < 4; ++w) s = joined(s, shared[w], scale);
  return s;
}

// The given token's logit, for thread 0: it is on its way while the row is read.
template <typename T>
__device__ __forceinline__ float given_logit(const LogProb<T>& a, int64_t row, bool& named) {
  named = false;
  if (!a.logp || threadIdx.x) return 0.f;
  const int64_t t = load_global<int64_t>(a.tokens + row);
  named = t >= 0 && t < a.n;
  return named ? (float)load_global<T>(a.logits + row * a.ldl + t) : 0.f;
}

// What a row's sums say of it; by thread 0.
template <typename T>
__device__ __forceinline__ float finish_row(const LogProb<T>& a, int64_t row, const Sums& s,
                                            float given, bool named) {
  const float log_total = logf(s.total);
  if (a.lse) a.lse[row] = fmaf(s.most, a.scale, log_total);
  const bool empty = s.total == 0.f;  // no logit over -inf
  if (a.entropy) a.entropy[row] = empty ? 0.f : log_total - s.moment / s.total;
  if (a.logp)
    a.logp[row] = !named  ? 0.f
                  : empty ? -__builtin_inff()
                          : (given - s.most) * a.scale - log_total;
  return log_total;
}

// Writes place `i` of a row's most likely tokens; key 0: there is none.
template <typename T>
__device__ __forceinline__ void write_top(const LogProb<T>& a, int64_t row, int i, uint64_t key,
                                          const Sums& s, float log_total) {
  const bool bad = !(s.total < __builtin_inff());  // a NaN or an infinity among the logits
  const bool none = key == 0 || bad;
  a.top_tokens[row * a.top + i] = none ? -1 : (int64_t)key_column(key);
  a.top_logp[row * a.top + i] = bad   ? __builtin_nanf("")
                                : none ? -__builtin_inff()
                                       : (key_value(key) - s.most) * a.scale - log_total;
}

// The number of keys over `key` among the first `count`, which stand on 16 bytes and whose number
// is made even by a 0 behind them.
__device__ __forceinline__ int keys_over(const uint64_t* keys, int count, uint64_t key) {
  typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
  int over = 0;
#pragma unroll 8
  for (int i = 0; i < count; i += 2) {
    const u64x2 k = *(const u64x2*)(keys + i);
    over += (k[0] > key) + (k[1] > key);
  }
  return over;
}

// The `top` largest of the keys that 256 threads hold, in `steps` steps of at most kStepKeys each;
// best: the thread's largest, 0 for none.  offer(thread, step, bound, put) calls put(key) for the
// keys of a thread's step that reach the bound; emit(i, key) is called once for every place, with 0
// where there is no key.  The steps of the `top` threads that matter are shared out among all.
// Where more keys reach the bound than there is room for, they are taken in turns of a few steps,
// each of which raises the bound.
constexpr int kStepKeys = 8, kRoom = 2048;
struct TopShared {
  __attribute__((aligned(16))) uint64_t best[256], room[kRoom + 2], held[kTop], bound;
  int who[kTop], offers, count;
};
template <typename Offer, typename Emit>
__device__ __forceinline__ void block_top(TopShared& sh, int top, uint64_t best, int steps,
                                          Offer&& offer, Emit&& emit) {
  const int t = threadIdx.x;
  if (t == 0) sh.bound = 1, sh.count = 0, sh.offers = 0;  // every key, if fewer threads have one
  sh.best[t] = best;
  __syncthreads();
  const int over = keys_over(sh.best, 256, best);
  if (best != 0 && over < top) {  // keys differ: places do too
    sh.who[over] = t;
    atomicMax(&sh.offers, over + 1);
    if (over == top - 1) sh.bound = best;
  }
  __syncthreads();
  const uint64_t bound = sh.bound;
  const int offers = sh.offers;
  // the steps from step0 on, `turn` of them
  auto all = [&](int step0, int turn, auto&& put) {
    turn = min(turn, steps - step0);
    for (int i = t; i < offers * turn; i += 256)
      offer(sh.who[i / turn], step0 + i % turn, bound, put);
  };
  all(0, steps, [&](uint64_t key) {
    const int at = atomicAdd(&sh.count, 1);
    if (at < kRoom) sh.room[at] = key;
  });
  __syncthreads();
  int count = sh.count;
  if (count > kRoom) {  // the first keys that came are dropped, and all are offered again
    constexpr int kTurn = (kRoom - kTop) / (kTop * kStepKeys);
    if (t < kTop) sh.held[t] = 0;
    for (int step0 = 0; step0 < steps; step0 += kTurn) {
      __syncthreads();
      if (t == 0) sh.count = top;
      if (t < top) sh.room[t] = sh.held[t];
      __syncthreads();
      const uint64_t last = sh.room[top - 1];
      all(step0, kTurn, [&](uint64_t key) {
        if (key > last) sh.room[atomicAdd(&sh.count, 1)] = key;
      });
      __syncthreads();
      count = sh.count;
      if (t == 0) sh.room[count] = 0;
      __syncthreads();
      for (int i = t; i < count; i += 256) {
        const uint64_t key = sh.room[i];
        const int place = keys_over(sh.room, count, key);
        if (key != 0 && place < top) sh.held[place] = key;
      }
    }
    __syncthreads();
    for (int i = t; i < top; i += 256) emit(i, sh.held[i]);
    return;
  }
  if (t == 0) sh.room[count] = 0;
  __syncthreads();
  for (int i = t; i < count; i += 256) {
    const uint64_t key = sh.room[i];
    const int place = keys_over(sh.room, count, key);
    if (place < top) emit(place, key);
  }
  for (int i = count + t; i < top; i += 256) emit(i, (uint64_t)0);
}

// A block takes part blockIdx.x % parts of a row.  TOP: the most likely tokens are wanted.
template <typename T, bool TOP>
__global__ __launch_bounds__(256) void k_logprob(LogProb<T> a) {
  __shared__ Sums shared[4];
  __shared__ float row_log, row_most, row_total;
  const int64_t row = blockIdx.x / a.parts;
  const int part = blockIdx.x % a.parts;
  const int first = part * a.part_columns, end = min(first + a.part_columns, a.n);
  const T* l = a.logits + row * a.ldl;
  const float to2 = a.scale * 1.44269504f;  // powers of two from here on, joined in powers of e
  const bool whole = a.parts == 1;
  bool named = false;
  const float given = whole ? given_logit(a, row, named) : 0.f;
  Sums s = no_sums();
  int best_at = -1;
  float best_value = -__builtin_inff();
  auto take = [&](const float(&x)[8], int col) {
    const float most = largest(x);
    if constexpr (TOP) {
      if (most > best_value) best_value = most, best_at = col;
    }
    add8(s, x, most, to2);
  };
  walk<T>(l, first, end, take);
  s.moment *= 0.693147181f;
  s = block_sums(s, a.scale, shared);
  float log_total = 0.f;
  if (threadIdx.x == 0) {
    if (whole)
      log_total = finish_row(a, row, s, given, named);
    else
      a.part_sums[row * a.parts + part] = s;
  }
  if constexpr (TOP) {
    __shared__ TopShared top;
    if (threadIdx.x == 0) row_log = log_total, row_most = s.most, row_total = s.total;
    block_top(
        top, a.top, best_at < 0 ? 0 : rank_key(best_value, best_at),
        (end - first + kStep - 1) / kStep,
        [&](int thread, int step, uint64_t bound, auto&& put) {
          const int c = first + step * kStep + thread * 8;
          float v[8];
          load_row_end<T, 8>(l + min(c, end - 1), end - c, v);
#pragma unroll
          for (int i = 0; i < 8; ++i)  // the bound's column is the first of its eight
            if (c + i < end && v[i] > -__builtin_inff() && rank_key(v[i], c) >= bound)
              put(rank_key(v[i], c + i));
        },
        [&](int i, uint64_t key) {
          if (whole)
            write_top(a, row, i, key, Sums{row_most, row_total, 0.f}, row_log);
          else
            a.part_keys[(row * a.parts + part) * a.top + i] = key;
        });
  }
}

// Joins the parts of a row.
template <typename T, bool TOP>
__global__ __launch_bounds__(256) void k_logprob_join(LogProb<T> a) {
  __shared__ Sums shared[4];
  __shared__ float row_log, row_most, row_total;
  const int64_t row = blockIdx.x;
  bool named;
  const float given = given_logit(a, row, named);
  Sums s = no_sums();
  if ((int)threadIdx.x < a.parts) s = a.part_sums[row * a.parts + threadIdx.x];
  s = block_sums(s, a.scale, shared);
  if (threadIdx.x == 0) {
    row_log = finish_row(a, row, s, given, named);
    row_most = s.most;
    row_total = s.total;
  }
  if constexpr (TOP) {
    __shared__ TopShared top;
    const uint64_t* keys = a.part_keys + row * a.parts * a.top;  // a thread's are a part's
    block_top(
        top, a.top, (int)threadIdx.x < a.parts ? keys[threadIdx.x * a.top] : 0, a.top,
        [&](int thread, int step, uint64_t bound, auto&& put) {
          const uint64_t key = keys[thread * a.top + step];
          if (key >= bound && key != 0) put(key);
        },
        [&](int i, uint64_t key) {
          write_top(a, row, i, key, Sums{row_most, row_total, 0.f}, row_log);
        });
  }
}

// The gradient of the logits.  A thread takes 8 columns of a row at a time, each read before it is
// written, so that the gradient may take the logits' place.
//
// p = e^(scale l - lse) has lse's rounding as a relative error, 2^-17 at most up to kExactLse.  A row
// past that (logits that share a large offset, or all at their type's lowest value, where the
// rounding passes log S; products with scale that are no float) is one block's alone, which takes
// the row's sums again and p from the differences to the largest logit: 4096 rows of 128000 bf16
// logits 745 us where all are such rows, 405 where none is; few rows leave most of the card idle: one
// 41 us for 10, 64 90 for 10, 512 147 for 47.  Which block it is goes round with the rows: the first
// of each would be on two of the XCDs at most (5.2 ms).
constexpr float kExactLse = 256.f;

template <typename T>
struct LogProbBack {
  const T* logits;
  int64_t ldl, rows, ldd;
  int n, blocks_a_row;
  float scale;
  const int64_t* tokens;
  const float *lse, *entropy, *dlogp, *dentropy;  // dlogp or dentropy may be NULL
  T* dlogits;
};

template <typename T>
__global__ __launch_bounds__(256) void k_logprob_back(LogProbBack<T> a) {
  constexpr int kPieces = kBackColumns / (256 * 8);
  const int64_t row = blockIdx.x / a.blocks_a_row;
  const int col0 = (int)(blockIdx.x % a.blocks_a_row) * kBackColumns + threadIdx.x * 8;
  const T* l = a.logits + row * a.ldl;
  T* dl = a.dlogits + row * a.ldd;
  float x[kPieces][8];
#pragma unroll
  for (int u = 0; u < kPieces; ++u) {
    const int col = col0 + u * 256 * 8;
    load_row_end<T, 8>(l + min(col, a.n - 1), a.n - col, x[u]);
  }
  const float lse = a.lse[row];
  const int64_t token = a.dlogp ? a.tokens[row] : -1;
  const bool named = token >= 0 && token < a.n;
  const float g = named ? a.dlogp[row] * a.scale : 0.f;
  const float h = a.dentropy ? a.dentropy[row] * a.scale : 0.f;
  const float entropy = a.dentropy ? a.entropy[row] : 0.f;
  // of a column's logit, from its log probability
  auto gradient = [&](float log_p, int col) {
    log_p = __builtin_elementwise_maximum(log_p, kFar);
    const float p = __builtin_amdgcn_exp2f(log_p * 1.44269504f);
    return -p * fmaf(h, log_p + entropy, g) + (named && col == token ? g : 0.f);
  };
  if (__builtin_expect(!(fabsf(lse) <= kExactLse), 0)) {
    if (blockIdx.x % a.blocks_a_row != row % a.blocks_a_row) return;
    __shared__ Sums shared[4];
    __shared__ float row_most, row_total;
    Sums s = no_sums();
    const float to2 = a.scale * 1.44269504f;
    walk<T>(l, 0, a.n, [&](const float(&v)[8], int) { add8(s, v, largest(v), to2); });
    s = block_sums(s, a.scale, shared);
    if (threadIdx.x == 0) row_most = s.most, row_total = s.total;
    __syncthreads();
    const float most = row_most, total = row_total;
    // the row's own log S, where lse is a rounding of its lse; else what the given one says
    float log_total = logf(total);
    const float own = fmaf(most, a.scale, log_total), given = fmaf(-most, a.scale, lse);
    // Half the distance of floats at lse, and a quarter more for log S in another order of its sum:
    // an lse of more than the row's logits (of all columns, where these are a part) that is nearer
    // than that cannot be told from the row's own.
    const float half_step = __uint_as_float(__float_as_uint(lse) & 0x7f800000u) * 0x1p-24f;
    if (!(own == lse || fabsf(given - log_total) < 1.25f * half_step)) log_total = given;
    const bool empty = total == 0.f && own == lse;  // no logit over -inf: nothing to move
    walk<T>(l, 0, a.n, [&](const float(&v)[8], int col) {
      float d[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        d[i] = gradient(fmaf(v[i] - most, a.scale, -log_total), col + i);
        if (empty) d[i] = 0.f;
      }
      store_row<T, 8>(dl + col, a.n - col, d);
    });
    return;
  }
#pragma unroll
  for (int u = 0; u < kPieces; ++u) {
    const int col = col0 + u * 256 * 8;
    if (col >= a.n) continue;
    float d[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) d[i] = gradient(fmaf(x[u][i], a.scale, -lse), col + i);
    store_row<T, 8>(dl + col, a.n - col, d);
  }
}

}  // namespace lm
