// The ends of a language model: host side of lirpa_embed_* and lirpa_logprob_*.  Kernels:
// embed.hpp, logprob.hpp.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "embed.hpp"
#include "lirpa.h"
#include "lm_host.hpp"
#include "logprob.hpp"

using namespace lirpa_host;
using namespace lm;

namespace {

int check_tokens(const char* who, const void* p) {
  if (!p) return fail(LIRPA_EINVAL, "%s: tokens is null", who);
  if ((uintptr_t)p % 8) return fail(LIRPA_EINVAL, "%s: tokens is not aligned to its type", who);
  return LIRPA_OK;
}

int check_vocab(const char* who, int vocab) {
  if (vocab < 1 || vocab > kMaxWidth)
    return fail(LIRPA_EINVAL, "%s: vocab %d is outside [1, 2^20]", who, vocab);
  return LIRPA_OK;
}

// ---------------------------------------------------------------------------------------------
// Embedding
// ---------------------------------------------------------------------------------------------
int64_t pieces8(int n) { return (n + 7) / 8; }

// Entries of a piece of the sums: few where there are few rows, more where a frequent token's
// pieces, which one block joins, would be many.  Sums and join of bf16 rows, us: 3000 x 1000 9 + 10
// with 8, 21 + 9 with 32; 16384 x 4096 34 + 15 with 16, 34 + 25 with 8; 60000 x 400 27 + 17 with
// 32, 20 + 43 with 8.
int sum_entries(int64_t rows) { return (int)std::clamp<int64_t>(rows >> 10 & ~7, 8, 32); }

constexpr int kRadixBlocks = 256, kRadixLeast = 1024;

// Up to so many columns 16 pieces share a block of the sums, 16 threads each; a block a piece
// otherwise (4000 x 100: 11 us, 25 with a block a piece; 60000 x 400 takes 27 either way with 64
// threads a piece).
constexpr int kNarrow = 128;

struct EmbedRoom {
  Named *a, *b;
  uint32_t* counts;
  float* part;
  size_t bytes;
};
EmbedRoom embed_room(int64_t rows, int n, void* base) {
  Carver ws{(char*)base};
  EmbedRoom r;
  r.a = (Named*)ws.take((size_t)rows * sizeof(Named));
  r.b = (Named*)ws.take((size_t)rows * sizeof(Named));
  r.counts = (uint32_t*)ws.take(((size_t)kRadixBlocks << kMaxDigit) * sizeof(uint32_t));
  // no less than sum_entries asks for with fewer rows: 8 entries a piece up to 2^14
  const int64_t pieces = (rows + 31) / 32 + std::min<int64_t>((rows + 7) / 8, 1 << 11);
  r.part = (float*)ws.take((size_t)pieces * 2 * n * sizeof(float));
  r.bytes = std::max<size_t>(256, ws.at);
  return r;
}

template <typename T>
int embed_forward(int64_t rows, int n, int vocab, const int64_t* tokens, const T* table,
                  int64_t ldt, float scale, T* out, int64_t ldo, hipStream_t st) {
  const int64_t each = max_blocks(256) * 256 / pieces8(n);
  for (int64_t r0 = 0; r0 < rows; r0 += each) {
    const int64_t r = std::min(each, rows - r0), blocks = (r * pieces8(n) + 255) / 256;
    TRY(launch_k("embed_forward", st, [&] {
      k_embed_fwd<T><<<(unsigned)blocks, 256, 0, st>>>(tokens + r0, table, ldt, r, n, vocab, scale,
                                                       out + r0 * ldo, ldo);
    }));
  }
  return LIRPA_OK;
}

// The fill of the gradient, in equal parts over `launches` launches.
template <typename T>
struct Fills {
  EmbedFill<T> fill;
  int64_t total = 0, each = 0;

  Fills(T* dtable, int64_t ldd, const T* base, int64_t ldb, int vocab, int n, int launches) {
    const bool flat = ldd == n && (!base || ldb == n) && (int64_t)vocab * n >= 8;
    fill = {dtable, base, ldd, ldb, 0, 0, (int64_t)vocab * n, flat ? 0 : n};
    if (base != dtable) total = flat ? (fill.values + 7) / 8 : vocab * pieces8(n);
    each = up((total + launches - 1) / launches, kFillPieces);
  }
  // The next part: the blocks that it takes.
  int64_t next() {
    fill.first = fill.end;
    fill.end = std::min(total, fill.end + each);
    return (fill.end - fill.first + kFillPieces - 1) / kFillPieces;
  }
};

template <typename T>
int embed_backward(int64_t rows, int n, int vocab, const int64_t* tokens, const T* dout,
                   int64_t lddo, float scale, const T* base, int64_t ldb, T* dtable, int64_t ldd,
                   void* ws, hipStream_t st) {
  const EmbedRoom room = embed_room(rows, n, ws);
  const bool radix = rows > kRankRows;
  int bits = 1;
  while (vocab >> bits) ++bits;  // of vocab itself, which stands for padding
  const int passes = radix ? (bits + kMaxDigit - 1) / kMaxDigit : 0;
  const int digit = radix ? (bits + passes - 1) / passes : 0;
  Fills<T> fills(dtable, ldd, base, ldb, vocab, n, radix ? 2 * passes : 1);

  EmbedSum<T> sum{};
  sum.dout = dout;
  sum.base = base;
  sum.dtable = dtable;
  sum.part = room.part;
  sum.lddo = lddo;
  sum.ldb = ldb;
  sum.ldd = ldd;
  sum.rows = rows;
  sum.each = sum_entries(rows);
  sum.pieces = (int)((rows + sum.each - 1) / sum.each);
  sum.n = n;
  sum.vocab = vocab;
  sum.scale = scale;
  const int tx = n <= kNarrow ? 16 : 256;
  const int64_t slabs = (n + tx * 8 - 1) / (tx * 8), join_slabs = (n + 511) / 512;
  const int64_t sum_blocks = (sum.pieces + 256 / tx - 1) / (256 / tx) * slabs;
  const int64_t join_blocks = (int64_t)(sum.pieces - 1) * join_slabs;
  if (std::max({sum_blocks, join_blocks, fills.each / kFillPieces + kRadixBlocks}) >
      max_blocks(256))
    return fail(LIRPA_EUNSUPPORTED, "lirpa_embed_backward: more than 2^35 values");

  const Named* named = room.a;
  if (!radix) {
    const int64_t sort = (rows + 63) / 64, blocks = sort + fills.next();
    if (blocks)
      TRY(launch_k("embed_sort", st, [&] {
        k_embed_rank<T><<<(unsigned)blocks, 256, 0, st>>>(tokens, (int)rows, vocab, room.a,
                                                          (int)sort, fills.fill);
      }));
  } else {
    RadixPass r{};
    r.tokens = tokens;
    r.counts = room.counts;
    r.rows = rows;
    r.each = (int)std::max<int64_t>(kRadixLeast, up((rows + kRadixBlocks - 1) / kRadixBlocks, 256));
    r.blocks = (int)((rows + r.each - 1) / r.each);
    r.vocab = vocab;
    r.bits = digit;
    for (int p = 0; p < passes; ++p) {
      r.shift = p * digit;
      r.in = p == 0 ? nullptr : named;
      r.out = p % 2 ? room.b : room.a;
      TRY(launch_k("embed_sort", st, [&] {
        const unsigned blocks = (unsigned)(r.blocks + fills.next());
        k_embed_count<T><<<blocks, 256, 0, st>>>(r, fills.fill);
      }));
      TRY(launch_k("embed_sort", st, [&] {
        const unsigned blocks = (unsigned)(r.blocks + fills.next());
        k_embed_place<T><<<blocks, 256, 0, st>>>(r, fills.fill);
      }));
      named = r.out;
    }
  }
  if (rows == 0) return LIRPA_OK;
  sum.named = named;
  TRY(launch_k("embed_sum", st, [&] {
    if (tx == 16)
      k_embed_sum<T, 16><<<(unsigned)sum_blocks, 256, 0, st>>>(sum, (int)slabs);
    else
      k_embed_sum<T, 256><<<(unsigned)sum_blocks, 256, 0, st>>>(sum, (int)slabs);
  }));
  if (join_blocks == 0) return LIRPA_OK;
  return launch_k("embed_join", st, [&] {
    k_embed_join<T><<<(unsigned)join_blocks, 256, 0, st>>>(sum, (int)join_slabs);
  });
}

// ---------------------------------------------------------------------------------------------
// Log probabilities
// ---------------------------------------------------------------------------------------------
// Few rows are split, so that about kFewBlocks blocks have work: rows * parts < 2 * kFewBlocks.  A
// part costs a launch that joins (6 us, 10 with alternatives) and, with alternatives, its own
// search (4 us): 61 rows of 50000 bf16 logits with 5 alternatives take 22 us in parts of about 256
// blocks, 24 of 1024 and 26 of 4096; 300 rows 19 us whole and 30 in four parts, 8000 logits without
// alternatives 8 and 13.
constexpr int kFewBlocks = 256;
void logprob_parts(int64_t rows, int n, int& parts, int& columns) {
  const int64_t most = std::min<int64_t>(kMaxParts, (n + kPartColumns - 1) / kPartColumns);
  const int64_t want = std::clamp<int64_t>((kFewBlocks + rows - 1) / rows, 1, most);
  columns = want == 1 ? n : (int)up((n + want - 1) / want, kPartColumns);
  parts = (n + columns - 1) / columns;
}

size_t logprob_bytes(int n, int top) {
  if (n <= kPartColumns) return 256;
  return up(2 * kFewBlocks * sizeof(Sums), 256) + (size_t)2 * kFewBlocks * top * sizeof(uint64_t);
}

template <typename T>
int logprob_forward(LogProb<T> a, void* ws, hipStream_t st) {
  logprob_parts(a.rows, a.n, a.parts, a.part_columns);
  if (a.parts > 1) {
    Carver c{(char*)ws};
    a.part_sums = (Sums*)c.take(2 * kFewBlocks * sizeof(Sums));
    a.part_keys = (uint64_t*)c.take((size_t)2 * kFewBlocks * a.top * sizeof(uint64_t));
  }
  const int64_t each = max_blocks(256) / a.parts;
  for (int64_t left = a.rows; left > 0; left -= each) {
    a.rows = std::min(each, left);
    const unsigned blocks = (unsigned)(a.rows * a.parts);
    TRY(launch_k("logprob", st, [&] {
      if (a.top)
        k_logprob<T, true><<<blocks, 256, 0, st>>>(a);
      else
        k_logprob<T, false><<<blocks, 256, 0, st>>>(a);
    }));
    if (a.parts > 1)
      TRY(launch_k("logprob_join", st, [&] {
        if (a.top)
          k_logprob_join<T, true><<<(unsigned)a.rows, 256, 0, st>>>(a);
        else
          k_logprob_join<T, false><<<(unsigned)a.rows, 256, 0, st>>>(a);
      }));
    a.logits += a.rows * a.ldl;
    if (a.tokens) a.tokens += a.rows;
    if (a.logp) a.logp += a.rows;
    if (a.lse) a.lse += a.rows;
    if (a.entropy) a.entropy += a.rows;
    if (a.top) {
      a.top_logp += a.rows * a.top;
      a.top_tokens += a.rows * a.top;
    }
  }
  return LIRPA_OK;
}

template <typename T>
int logprob_backward(LogProbBack<T> a, hipStream_t st) {
  a.blocks_a_row = (a.n + kBackColumns - 1) / kBackColumns;
  const int64_t each = max_blocks(256) / a.blocks_a_row;
  for (int64_t left = a.rows; left > 0; left -= each) {
    a.rows = std::min(each, left);
    TRY(launch_k("logprob_backward", st, [&] {
      k_logprob_back<T><<<(unsigned)(a.rows * a.blocks_a_row), 256, 0, st>>>(a);
    }));
    a.logits += a.rows * a.ldl;
    a.dlogits += a.rows * a.ldd;
    a.lse += a.rows;
    if (a.tokens) a.tokens += a.rows;
    if (a.entropy) a.entropy += a.rows;
    if (a.dlogp) a.dlogp += a.rows;
    if (a.dentropy) a.dentropy += a.rows;
  }
  return LIRPA_OK;
}

int check_scale(const char* who, float scale) {
  if (!std::isfinite(scale)) return fail(LIRPA_EINVAL, "%s: scale must be finite", who);
  return LIRPA_OK;
}

// Of logits: its product with 1 / log 2 is a float too.
int check_factor(const char* who, float scale) {
  if (!(scale > 0.f) || scale > 0x1p100f)
    return fail(LIRPA_EINVAL, "%s: scale must be over 0 and at most 2^100", who);
  return LIRPA_OK;
}

}  // namespace

extern "C" {

int lirpa_embed_forward(int dtype, int64_t rows, int n, int vocab, const int64_t* tokens,
                        const void* table, int64_t ldt, float scale, void* out, int64_t ldo,
                        hipStream_t stream) {
  return guarded([&] {
    const char* who = "lirpa_embed_forward";
    TRY(check_shape(who, dtype, rows, n));
    TRY(check_vocab(who, vocab));
    TRY(check_scale(who, scale));
    if (rows == 0) return (int)LIRPA_OK;
    TRY(check_tokens(who, tokens));
    TRY(check_rows(who, "table", dtype, table, ldt, n));
    TRY(check_rows(who, "out", dtype, out, ldo, n));
    return by_type(dtype, [&](auto t) {
      using T = decltype(t);
      return embed_forward<T>(rows, n, vocab, tokens, (const T*)table, ldt, scale, (T*)out, ldo,
                              stream);
    });
  });
}

size_t lirpa_embed_workspace_bytes(int64_t rows, int n) {
  if (rows < 0 || rows > kMaxRows || n < 1 || n > kMaxWidth) return 0;
  return embed_room(rows, n, nullptr).bytes;
}

int lirpa_embed_backward(int dtype, int64_t rows, int n, int vocab, const int64_t* tokens,
                         const void* dout, int64_t lddo, float scale, const void* base, int64_t ldb,
                         void* dtable, int64_t ldd, void* ws, size_t ws_bytes,
                         hipStream_t stream) {
  return guarded([&] {
    const char* who = "lirpa_embed_backward";
    TRY(check_shape(who, dtype, rows, n));
    TRY(check_vocab(who, vocab));
    TRY(check_scale(who, scale));
    if (rows > 0) {
      TRY(check_tokens(who, tokens));
      TRY(check_rows(who, "dout", dtype, dout, lddo, n));
    }
    if (base) TRY(check_rows(who, "base", dtype, base, ldb, n));
    TRY(check_rows(who, "dtable", dtype, dtable, ldd, n));
    TRY(check_in_place(who, "dtable", dtable, ldd, "base", base, ldb, vocab));
    TRY(check_ws(who, ws, ws_bytes, lirpa_embed_workspace_bytes(rows, n)));
    return by_type(dtype, [&](auto t) {
      using T = decltype(t);
      return embed_backward<T>(rows, n, vocab, tokens, (const T*)dout, lddo, scale, (const T*)base,
                               ldb, (T*)dtable, ldd, ws, stream);
    });
  });
}

size_t lirpa_logprob_workspace_bytes(int64_t rows, int n, int top) {
  if (rows < 0 || rows > kMaxRows || n < 1 || n > kMaxWidth || top < 0 || top > kTop) return 0;
  return logprob_bytes(n, top);
}

int lirpa_logprob_forward(int dtype, int64_t rows, int n, const void* logits, int64_t ldl,
                          float scale, const int64_t* tokens, float* logp, float* lse,
                          float* entropy, int top, float* top_logp, int64_t* top_tokens, void* ws,
                          size_t ws_bytes, hipStream_t stream) {
  return guarded([&] {
    const char* who = "lirpa_logprob_forward";
    TRY(check_shape(who, dtype, rows, n));
    TRY(check_factor(who, scale));
    if (top < 0 || top > kTop)
      return fail(LIRPA_EINVAL, "%s: top = %d is outside [0, %d]", who, top, kTop);
    if (rows == 0) return (int)LIRPA_OK;
    if (!logp && !lse && !entropy && !top)
      return fail(LIRPA_EINVAL, "%s: no output is wanted", who);
    TRY(check_rows(who, "logits", dtype, logits, ldl, n));
    if (logp) TRY(check_tokens(who, tokens));
    TRY(check_floats(who, "logp", logp));
    TRY(check_floats(who, "lse", lse));
    TRY(check_floats(who, "entropy", entropy));
    if (top) {
      if (!top_logp || !top_tokens)
        return fail(LIRPA_EINVAL, "%s: top_logp or top_tokens is null", who);
      TRY(check_floats(who, "top_logp", top_logp));
      if ((uintptr_t)top_tokens % 8)
        return fail(LIRPA_EINVAL, "%s: top_tokens is not aligned to its type", who);
    }
    TRY(check_ws(who, ws, ws_bytes, lirpa_logprob_workspace_bytes(rows, n, top)));
    return by_type(dtype, [&](auto t) {
      using T = decltype(t);
      LogProb<T> a{};
      a.logits = (const T*)logits;
      a.ldl = ldl;
      a.rows = rows;
      a.n = n;
      a.top = top;
      a.scale = scale;
      a.tokens = tokens;
      a.logp = logp;
      a.lse = lse;
      a.entropy = entropy;
      a.top_logp = top_logp;
      a.top_tokens = top_tokens;
      return logprob_forward(a, ws, stream);
    });
  });
}

int lirpa_logprob_backward(int dtype, int64_t rows, int n, const void* logits, int64_t ldl,
                           float scale, const int64_t* tokens, const float* lse,
                           const float* entropy, const float* dlogp, const float* dentropy,
                           void* dlogits, int64_t ldd, hipStream_t stream) {
  return guarded([&] {
    const char* who = "lirpa_logprob_backward";
    TRY(check_shape(who, dtype, rows, n));
    TRY(check_factor(who, scale));
    if (rows == 0) return (int)LIRPA_OK;
    if (!dlogp && !dentropy) return fail(LIRPA_EINVAL, "%s: no gradient comes in", who);
    TRY(check_rows(who, "logits", dtype, logits, ldl, n));
    TRY(check_rows(who, "dlogits", dtype, dlogits, ldd, n));
    TRY(check_in_place(who, "dlogits", dlogits, ldd, "logits", logits, ldl, rows));
    if (!lse) return fail(LIRPA_EINVAL, "%s: lse is null", who);
    TRY(check_floats(who, "lse", lse));
    if (dlogp) TRY(check_tokens(who, tokens));
    TRY(check_floats(who, "dlogp", dlogp));
    if (dentropy && !entropy) return fail(LIRPA_EINVAL, "%s: entropy is null", who);
    TRY(check_floats(who, "entropy", entropy));
    TRY(check_floats(who, "dentropy", dentropy));
    return by_type(dtype, [&](auto t) {
      using T = decltype(t);
      LogProbBack<T> a{};
      a.logits = (const T*)logits;
      a.ldl = ldl;
      a.rows = rows;
      a.ldd = ldd;
      a.n = n;
      a.scale = scale;
      a.tokens = tokens;
      a.lse = lse;
      a.entropy = entropy;
      a.dlogp = dlogp;
      a.dentropy = dentropy;
      a.dlogits = (T*)dlogits;
      return logprob_backward(a, stream);
    });
  });
}

}  // extern "C"
