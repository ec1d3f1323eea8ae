// The feed-forward block of a language model: host side of lirpa_q8_*, lirpa_norm_* and
// lirpa_ffn_*.  Kernels: q8.hpp, norm.hpp, ffn_tile.hpp, ffn_few.hpp.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ffn_few.hpp"
#include "ffn_tile.hpp"
#include "lirpa.h"
#include "lm_host.hpp"
#include "norm.hpp"
#include "q8.hpp"

using namespace lirpa_host;
using namespace lm;

namespace {

// ---------------------------------------------------------------------------------------------
// 8 bits
// ---------------------------------------------------------------------------------------------
int64_t q8_exps_at(int64_t rows, int n) { return rows * groups_of(n) * kGroup; }
size_t q8_bytes(int64_t rows, int n) { return (size_t)rows * groups_of(n) * (kGroup + 1); }

int check_q8(const char* who, const char* what, const void* p) {
  if (!p) return fail(LIRPA_EINVAL, "%s: %s is null", who, what);
  if (!aligned16(p)) return fail(LIRPA_EINVAL, "%s: %s does not start on 16 bytes", who, what);
  return LIRPA_OK;
}

// Rows of groups that one launch takes, a thread for 8 columns; more go out in several.
int64_t q8_launch_rows(int n) { return max_blocks(256) * 256 / (groups_of(n) * 4); }

template <typename T>
int q8_pack(int64_t rows, int n, const T* x, int64_t ldx, void* q8, hipStream_t st) {
  const int64_t each = q8_launch_rows(n), groups = groups_of(n);
  for (int64_t r0 = 0; r0 < rows; r0 += each) {
    const int64_t r = std::min(each, rows - r0), blocks = (r * groups * 4 + 255) / 256;
    TRY(launch_k("q8_pack", st, [&] {
      k_q8_pack<T><<<(unsigned)blocks, 256, 0, st>>>(
          x + r0 * ldx, ldx, r, n, (int8_t*)q8 + r0 * groups * kGroup,
          (uint8_t*)q8 + q8_exps_at(rows, n) + r0 * groups);
    }));
  }
  return LIRPA_OK;
}

template <typename T>
int q8_unpack(int64_t rows, int n, const void* q8, T* x, int64_t ldx, hipStream_t st) {
  const int64_t each = q8_launch_rows(n), groups = groups_of(n);
  for (int64_t r0 = 0; r0 < rows; r0 += each) {
    const int64_t r = std::min(each, rows - r0), blocks = (r * groups * 4 + 255) / 256;
    TRY(launch_k("q8_unpack", st, [&] {
      k_q8_unpack<T><<<(unsigned)blocks, 256, 0, st>>>(
          (const int8_t*)q8 + r0 * groups * kGroup,
          (const uint8_t*)q8 + q8_exps_at(rows, n) + r0 * groups, r, n, x + r0 * ldx, ldx);
    }));
  }
  return LIRPA_OK;
}

// ---------------------------------------------------------------------------------------------
// Norm
// ---------------------------------------------------------------------------------------------
// Threads a row and pieces of 8 columns a thread: one wave up to 2048 columns, then a block.  Rows
// over 16384 columns are read twice: with four pieces the backward pass does not fit the registers
// of 1024 threads.
struct NormShape {
  int threads, ch;
};
NormShape norm_shape(int n) {
  const int pieces = (n + 7) / 8;
  for (NormShape s : {NormShape{64, 1}, {64, 2}, {64, 4}, {256, 2}, {256, 4}, {1024, 2}})
    if (pieces <= s.threads * s.ch) return s;
  return {1024, 0};
}

template <typename F>
int by_norm_shape(NormShape s, F&& f) {
  using std::integral_constant;
#define SHAPE(T, C) \
  if (s.threads == T && s.ch == C) return f(integral_constant<int, T>{}, integral_constant<int, C>{})
  SHAPE(64, 1);
  SHAPE(64, 2);
  SHAPE(64, 4);
  SHAPE(256, 2);
  SHAPE(256, 4);
  SHAPE(1024, 2);
#undef SHAPE
  return f(integral_constant<int, 1024>{}, integral_constant<int, 0>{});
}

template <typename T>
int norm_fwd(NormFwd<T> a, hipStream_t st) {
  const NormShape s = norm_shape(a.n);
  const int per_block = s.threads == 64 ? 4 : 1, threads = s.threads == 64 ? 256 : s.threads;
  const int64_t each = max_blocks(threads) * per_block;  // rows a launch
  for (int64_t left = a.rows; left > 0; left -= each) {
    a.rows = std::min(each, left);
    const int64_t blocks = (a.rows + per_block - 1) / per_block;
    TRY(by_norm_shape(s, [&](auto th, auto ch) {
      return launch_k("norm_forward", st, [&] {
        k_norm_fwd<T, th.value, ch.value><<<(unsigned)blocks, threads, 0, st>>>(a);
      });
    }));
    a.x += a.rows * a.ldx;
    if (a.res) a.res += a.rows * a.ldr;
    if (a.sum) a.sum += a.rows * a.lds;
    if (a.y) a.y += a.rows * a.ldy;
    if (a.q) {
      a.q += a.rows * groups_of(a.n) * kGroup;
      a.exps += a.rows * groups_of(a.n);
    }
    if (a.rstd) a.rstd += a.rows;
  }
  return LIRPA_OK;
}

// Blocks of the backward pass, and so partial sums of dw: enough to fill the chip.
int64_t norm_bwd_blocks(int64_t rows, int n) {
  const NormShape s = norm_shape(n);
  const int64_t units = s.threads == 64 ? (rows + 3) / 4 : rows;
  return std::min<int64_t>(units, s.threads == 64 ? 1024 : s.threads == 256 ? 1024 : 512);
}

template <typename T>
int norm_bwd(NormBwd<T> a, T* dw, float* part, hipStream_t st) {
  const NormShape s = norm_shape(a.n);
  const int64_t blocks = norm_bwd_blocks(a.rows, a.n);
  a.part = dw ? part : nullptr;
  // dw of wide rows has a kernel of its own, which reads dy before dh may take its place
  if (dw && blocks > 0 && s.ch == 0)
    TRY(launch_k("norm_backward", st, [&] {
      k_norm_dw_wide<T><<<dim3((a.n + 2047) / 2048, (unsigned)blocks), 256, 0, st>>>(a);
    }));
  if (blocks > 0 && (a.dh || s.ch > 0)) {
    TRY(by_norm_shape(s, [&](auto th, auto ch) {
      return launch_k("norm_backward", st, [&] {
        const unsigned threads = th.value == 64 ? 256 : th.value;
        if (ch.value == 0 || a.n % 8)
          k_norm_bwd<T, th.value, ch.value, true><<<(unsigned)blocks, threads, 0, st>>>(a);
        else if constexpr (ch.value > 0)
          k_norm_bwd<T, th.value, ch.value, false><<<(unsigned)blocks, threads, 0, st>>>(a);
      });
    }));
  }
  if (dw)
    TRY(launch_k("norm_dw", st, [&] {
      k_norm_dw<T><<<(a.n + 31) / 32, 256, 0, st>>>(part, (int)blocks, a.n, dw);
    }));
  return LIRPA_OK;
}

// ---------------------------------------------------------------------------------------------
// Feed-forward block
// ---------------------------------------------------------------------------------------------
int check_ffn(const char* who, const lirpa_ffn* f) {
  if (!f) return fail(LIRPA_EINVAL, "%s: the block is null", who);
  TRY(check_shape(who, f->dtype, 0, f->n_model));
  TRY(check_shape(who, f->dtype, 0, f->n_hidden));
  if (f->gate != LIRPA_GATE_RELU && f->gate != LIRPA_GATE_SILU && f->gate != LIRPA_GATE_GELU)
    return fail(LIRPA_EINVAL, "%s: gate %d is none of lirpa_gate", who, f->gate);
  TRY(check_rows(who, "Wg", f->dtype, f->Wg, f->ldg, f->n_model));
  TRY(check_rows(who, "Wu", f->dtype, f->Wu, f->ldu, f->n_model));
  TRY(check_rows(who, "Wd", f->dtype, f->Wd, f->ldd, f->n_hidden));
  return LIRPA_OK;
}

// An operand of the tile kernel: 16 bits, rows on 16 bytes, length a multiple of 8 or padded to
// one with zeros.  `ld` in elements; parts of a 32-bit operand lie `plane` elements apart.
struct Operand {
  const char* p = nullptr;
  int64_t ld = 0, plane = 0;
};

struct FfnPlan {
  const lirpa_ffn* f;
  int64_t rows;
  bool f32;
  int parts;
  int64_t D, F, Dp, Fp;  // widths, and padded to 8
  Carver ws;

  FfnPlan(const lirpa_ffn* ffn, int64_t r, void* base)
      : f(ffn), rows(r), f32(ffn->dtype == LIRPA_F32), parts(f32 ? 3 : 1), D(ffn->n_model),
        F(ffn->n_hidden), Dp(up(D, 8)), Fp(up(F, 8)), ws{(char*)base} {}

  // Room for an operand of the library's own.
  Operand own(int64_t r, int64_t cols) {
    Operand o;
    o.ld = up(cols, 8);
    o.plane = r * o.ld;
    o.p = (const char*)ws.take((size_t)(parts * o.plane) * 2);
    return o;
  }
  bool in_place(const void* p, int64_t ld, int64_t cols) const {
    return !f32 && aligned16(p) && ld % 8 == 0 && cols % 8 == 0;
  }
  // Wg and Wu are read side by side, with one row distance.
  bool in_in_place() const {
    return in_place(f->Wg, f->ldg, D) && in_place(f->Wu, f->ldu, D) && f->ldg == f->ldu;
  }
  bool down_in_place() const { return in_place(f->Wd, f->ldd, F); }
};

// The operands that the tile kernel cannot read in place, copied into their rooms by one launch.
struct Copies {
  OperandJobs jobs{};
  int64_t blocks = 0;

  void add(bool in_place, const void* x, int64_t ldx, int64_t rows, int64_t n, Operand& o) {
    if (in_place) {
      o.p = (const char*)x;
      o.ld = ldx;
      o.plane = 0;
    } else {
      job(x, nullptr, ldx, rows, n, o);
    }
  }
  void add_packed(const void* q8, int64_t rows, int64_t n, const Operand& o) {
    job(q8, (const uint8_t*)q8 + q8_exps_at(rows, (int)n), 0, rows, n, o);
  }
  void job(const void* x, const uint8_t* exps, int64_t ldx, int64_t rows, int64_t n,
           const Operand& o) {
    if (rows == 0) return;
    jobs.job[jobs.count++] = {x, exps, ldx, rows, o.plane, (void*)o.p, (int)n, (int)o.ld,
                              (unsigned)blocks};
    blocks += (rows * (o.ld / 8) + 255) / 256;
  }
  int run(const FfnPlan& pl, hipStream_t st) const {
    if (blocks == 0) return LIRPA_OK;
    if (blocks > max_blocks(256))
      return fail(LIRPA_EUNSUPPORTED, "ffn_operands: more than 2^35 values");
    return launch_k("ffn_operands", st, [&] {
      switch (pl.f->dtype) {
        case LIRPA_F32: k_ffn_operands<Split><<<(unsigned)blocks, 256, 0, st>>>(jobs); break;
        case LIRPA_BF16: k_ffn_operands<bf16><<<(unsigned)blocks, 256, 0, st>>>(jobs); break;
        default: k_ffn_operands<f16><<<(unsigned)blocks, 256, 0, st>>>(jobs);
      }
    });
  }
};

// Parts (A, B) of the six products of 32-bit operands, smallest first.
constexpr int kSixA[6] = {1, 0, 2, 0, 1, 0};
constexpr int kSixB[6] = {1, 2, 0, 1, 0, 0};

// A product without its segments and output.
TileProblem problem(int64_t I, int64_t J, int64_t KA, int64_t KB) {
  TileProblem p{};
  p.I = (int)I;
  p.J = (int)J;
  p.KA = (int)KA;
  p.KB = (int)KB;
  p.splits = 1;
  return p;
}

// Adds the segments of one product.  `one_part`: A is exact in its first part.
void add_segs(const FfnPlan& pl, TileProblem& p, const Operand& A, const Operand& B,
              bool one_part = false) {
  const int n = !pl.f32 ? 1 : one_part ? 3 : 6;
  for (int s = 0; s < n; ++s) {
    const int64_t pa = n == 6 ? kSixA[s] : 0, pb = n == 6 ? kSixB[s] : n == 3 ? 2 - s : 0;
    p.A[p.nseg] = A.p + pa * 2 * A.plane;
    p.B[p.nseg++] = B.p + pb * 2 * B.plane;
  }
  p.lda = A.ld * 2;
  p.ldb = B.ld * 2;
}

TileArgs tile_args(const FfnPlan& pl, int keep) {
  TileArgs t{};
  t.count = 1;
  t.keep = keep;
  t.gate = pl.f->gate;
  return t;
}

// How a product is cut: tiles of 256 x 256 (one block a CU), 128 x 128 or 64 x 64 (two), and the
// number of blocks that share a tile's k, whose sums are then added by k_ffn_join.
struct Cut {
  int size = 128;
  int splits[kMaxProblems] = {1, 1, 1, 1};
};

// What a round of blocks over the 256 CUs takes: fixed + slope * k us for k in thousands, when it
// is full and when it is at most half full, and what the other epilogues add.  Measured at k = 64
// to 4096 in bf16; a full round computes 1, 2 and 4 tiles of 128 x 128 a CU.
struct Round {
  int size, full;  // tile, blocks
  double fixed, slope, half_fixed, half_slope, gate, back;
};
constexpr Round kRounds[3] = {{64, 1024, 6.0, 11.8, 4.5, 7.4, 1, 4},
                              {128, 512, 8.0, 14.3, 6.0, 8.7, 4.5, 12},
                              {256, 256, 10.0, 23.5, 10.0, 23.5, 8.6, 30}};

// The cut of least estimated time for the products of a launch.  Joining moves the sums twice at
// 4 TB/s and costs a launch (5 us; 10 with an epilogue, which then reads memory cold).  So few
// tiles over a long k are split, and tiles that would leave a round nearly empty, or most of its
// time to epilogues, are made smaller.
//
// Up to 64 tokens (`few`: both operands k-contiguous) it is the weights' bytes that count: tiles of
// 64, three more on their way, two blocks a CU.  4096 x 10944 in bf16: gate and up 34 us against
// 39-43 with tiles of 128, down 17 us in 8 parts, 22 in 4, 19 in 16.
int64_t tiles_of(const TileProblem& p, int64_t size, bool gate) {
  const int64_t feat = gate ? size / 2 : size;
  return (up(p.I, feat) / feat) * (up(p.J, size) / size);
}
int64_t steps_of(const TileProblem& p) {
  return up(std::max(p.KA, p.KB), kBK) / kBK * p.nseg;
}

int64_t part_ld(int64_t I) { return up(I, 8); }

// Room for the sums of products that are split.
size_t part_bytes(int splits, const TileProblem& p, int arrays) {
  return splits > 1 ? up((size_t)splits * arrays * p.J * part_ld(p.I) * sizeof(float), 256) : 0;
}
size_t part_room(const Cut& c, const TileProblem* probs, int count, int arrays = 1) {
  size_t bytes = 0;
  for (int i = 0; i < count; ++i) bytes += part_bytes(c.splits[i], probs[i], arrays);
  return bytes;
}

// The room that a call keeps for such sums.  It never falls with the rows, so that a workspace for
// many rows holds fewer too, and a cut that needs more is not taken: the most parts there can be,
// and no more than kMostParts.  Of 60,000 products up to 8192 rows of 4096 x 10944, that limit
// changes no cut of 16-bit types and 0.1 % of those of floats, whose estimated times grow by 1 % on
// average.
constexpr size_t kMostParts = (size_t)128 << 20, kMostParts32 = (size_t)256 << 20;
constexpr int kMaxSplits = 16;
size_t most_part_room(const FfnPlan& pl, const TileProblem* probs, int count, int arrays = 1) {
  int64_t longest = 1;
  for (int i = 0; i < count; ++i) longest = std::max(longest, steps_of(probs[i]));
  size_t bytes = 0;
  for (int i = 0; i < count; ++i) {
    const int64_t splits = std::min<int64_t>({kMaxSplits, longest / 4, steps_of(probs[i])});
    bytes += part_bytes((int)splits, probs[i], arrays);
  }
  return std::min(bytes, pl.f32 ? kMostParts32 : kMostParts);
}

// `may_large`: not the epilogue of da in 32 bits, which does not fit the larger tile's registers.
// `room`: for the sums of split products.
Cut cut_of(const TileProblem* probs, int count, int epi, bool may_large, bool few, size_t room) {
  const bool gate = epi == EPI_GATE;
  int64_t steps[kMaxProblems], longest = 1;
  for (int i = 0; i < count; ++i) {
    steps[i] = steps_of(probs[i]);
    longest = std::max(longest, steps[i]);
  }
  const bool weights = few && probs[0].J <= 64;
  Cut best;
  double least = 1e300;
  for (const Round& r : kRounds) {
    if (r.size == 256 && !may_large) continue;
    if (r.size > 64 && weights) continue;
    // tiles of 64 of two k-contiguous operands: two blocks a CU, more on their way (6.2 us at
    // most half full)
    const int full = r.size == 64 && few ? r.full / 2 : r.full;
    const double fixed = full < r.full ? r.half_fixed : r.fixed;
    const double slope = full < r.full ? r.half_slope : r.slope;
    const double more = gate ? r.gate : epi == EPI_BACK ? r.back : 0;
    int64_t tiles[kMaxProblems];
    for (int i = 0; i < count; ++i) tiles[i] = tiles_of(probs[i], r.size, gate);
    for (int parts : {1, 2, 3, 4, 5, 6, 8, 10, 12, kMaxSplits}) {
      if (parts > 1 && (longest < 4 * parts || (r.size == 256 && epi != EPI_STORE))) break;
      // blocks of about as many steps each, whichever product they are of
      const int64_t target = (longest + parts - 1) / parts;
      Cut c;
      c.size = r.size;
      int64_t blocks = 0;
      double sums = 0, k[kMaxProblems], longest_k = 0, shortest_k = 1e9;
      for (int i = 0; i < count; ++i) {
        c.splits[i] = (int)std::max<int64_t>(1, (steps[i] + target - 1) / target);
        k[i] = (double)((steps[i] + c.splits[i] - 1) / c.splits[i]) * kBK / 1024.0;
        longest_k = std::max(longest_k, k[i]);
        shortest_k = std::min(shortest_k, k[i]);
        blocks += tiles[i] * c.splits[i];
        if (c.splits[i] > 1)
          sums += (double)probs[i].I * probs[i].J * (gate ? 2 : 1) * c.splits[i];
      }
      if (part_room(c, probs, count, gate ? 2 : 1) > room) continue;
      const double base = fixed + (sums > 0 ? 0 : more);
      const double half = r.half_fixed + (sums > 0 ? 0 : more) +
                          (full < r.full ? 6.2 : r.half_slope) * longest_k;
      const int64_t whole = blocks / full, rest = blocks % full;
      double t;
      if (blocks <= full / 2) {
        t = half;
      } else if (longest_k == shortest_k || blocks <= full) {
        t = (double)whole * (base + slope * longest_k);
        if (rest > full / 2)
          t += base + slope * longest_k;
        else if (rest > 0)
          t += half;
      } else {  // blocks of several lengths, the shortest last: half of one is lost at the end
        t = 0.5 * (base + slope * shortest_k);
        for (int i = 0; i < count; ++i)
          t += (double)(tiles[i] * c.splits[i]) / full * (base + slope * k[i]);
        t = std::max(t, base + slope * longest_k);
      }
      if (sums > 0) t += (epi == EPI_STORE ? 5 : 10) + more + sums * 4 * 2 / 4e6;
      if (t < least) {
        least = t;
        best = c;
      }
    }
  }
  return best;
}

// Takes a product's split and its part of the room.
void split(TileProblem& p, int splits, char*& part, int arrays = 1) {
  p.splits = splits;
  if (splits == 1) return;
  p.part = (float*)part;
  p.part_ld = part_ld(p.I);
  part += part_bytes(splits, p, arrays);
}

// What the split products of a call leave to be added.
struct Joins {
  JoinJobs jobs{};
  int64_t blocks = 0;

  void add(const TileProblem& p) {
    jobs.job[jobs.count++] = {p.part, p.out, p.part_ld, p.ldo, p.J, p.I, p.splits,
                              (unsigned)blocks};
    blocks += ((int64_t)p.J * ((p.I + 7) / 8) + 255) / 256;
  }
  int run(const FfnPlan& pl, hipStream_t st) const {
    if (blocks == 0) return LIRPA_OK;
    if (blocks > max_blocks(256))
      return fail(LIRPA_EUNSUPPORTED, "ffn_join: more than 2^35 values");
    return launch_k("ffn_join", st, [&] {
      switch (pl.f->dtype) {
        case LIRPA_F32: k_ffn_join<float><<<(unsigned)blocks, 256, 0, st>>>(jobs); break;
        case LIRPA_BF16: k_ffn_join<bf16><<<(unsigned)blocks, 256, 0, st>>>(jobs); break;
        default: k_ffn_join<f16><<<(unsigned)blocks, 256, 0, st>>>(jobs);
      }
    });
  }
};

// Numbers the tiles; `total` blocks of `threads`.
template <int SIZE, int EPI>
int lay_out(const char* name, TileArgs& t, int threads, int64_t& total) {
  total = 0;
  for (int i = 0; i < t.count; ++i) {
    TileProblem& p = t.prob[i];
    const int64_t feat = EPI == EPI_GATE ? SIZE / 2 : SIZE;
    const int64_t ti = up(p.I, feat) / feat, tj = up(p.J, SIZE) / SIZE;
    if (total + ti * tj * p.splits > max_blocks(threads))
      return fail(LIRPA_EUNSUPPORTED, "%s: more than %lld tiles", name,
                  (long long)max_blocks(threads));
    p.tiles_i = (int)ti;
    p.tiles_j = (int)tj;
    p.first = (unsigned)total;
    total += ti * tj * p.splits;
  }
  return LIRPA_OK;
}

template <typename T, bool AKS, bool BKS, int EPI, int KEEP, int SIZE, int WI, int WJ, int AHEAD>
int launch_tile(const char* name, TileArgs& t, hipStream_t st) {
  int64_t total;
  TRY((lay_out<SIZE, EPI>(name, t, WI * WJ * 64, total)));
  if (total == 0) return LIRPA_OK;
  return launch_k(name, st, [&] {
    k_ffn_tile<T, AKS, BKS, EPI, KEEP, SIZE, WI, WJ, AHEAD>
        <<<(unsigned)total, WI * WJ * 64, 0, st>>>(t);
  });
}

template <typename T, bool AKS, bool BKS, int EPI, int KEEP>
int tile_of_size(const char* name, TileArgs& t, const Cut& c, char* part, Joins* joins,
                 hipStream_t st) {
  TileProblem& p = t.prob[0];
  split(p, c.splits[0], part, EPI == EPI_GATE ? 2 : 1);
  if (EPI == EPI_STORE && p.splits > 1) joins->add(p);
  if (c.size == 64) {
    // k-contiguous: for few tokens, where three more tiles on their way are worth their LDS
    constexpr int kAhead = !AKS && !BKS ? 3 : 1;
    TRY((launch_tile<T, AKS, BKS, EPI, KEEP, 64, 1, 4, kAhead>(name, t, st)));
  } else if (c.size == 128) {
    TRY((launch_tile<T, AKS, BKS, EPI, KEEP, 128, 2, 2, 1>(name, t, st)));
  } else {
    if constexpr (!(Kind<T>::kParts == 3 && EPI == EPI_BACK))
      TRY((launch_tile<T, AKS, BKS, EPI, KEEP, 256, 2, 4, 1>(name, t, st)));
  }
  if constexpr (EPI != EPI_STORE) {
    if (p.splits > 1) {
      const int64_t blocks = ((int64_t)p.J * groups_of(p.I) * 4 + 255) / 256;
      if (blocks == 0) return LIRPA_OK;
      if (blocks > max_blocks(256))
        return fail(LIRPA_EUNSUPPORTED, "ffn_finish: more than 2^35 values");
      return launch_k("ffn_finish", st, [&] {
        k_ffn_finish<T, EPI, KEEP><<<(unsigned)blocks, 256, 0, st>>>(t);
      });
    }
  }
  return LIRPA_OK;
}

template <typename T, int SIZE, int WI, int WJ>
int launch_grads(TileArgs& t, hipStream_t st) {
  int64_t total;
  TRY((lay_out<SIZE, EPI_STORE>("ffn_grads", t, WI * WJ * 64, total)));
  if (total == 0) return LIRPA_OK;
  return launch_k("ffn_grads", st, [&] {
    k_ffn_grads<T, SIZE, WI, WJ><<<(unsigned)total, WI * WJ * 64, 0, st>>>(t);
  });
}
template <typename T>
int grads_of_size(TileArgs& t, int size, hipStream_t st) {
  if (size == 64) return launch_grads<T, 64, 1, 4>(t, st);
  if (size == 128) return launch_grads<T, 128, 2, 2>(t, st);
  return launch_grads<T, 256, 2, 4>(t, st);
}
// All in one launch.  dx by itself gains 1 to 2 % where its tiles are whole rounds of the CUs
// (12,288 and 16,384 tokens of 4096 x 10944 in bf16: 4.42 and 5.99 ms, 4.46 and 6.05 together; 8192
// the same) and loses up to 12 % where they are not (8448: 3.31 ms, 2.96).
int run_grads(const FfnPlan& pl, TileArgs& t, int size, hipStream_t st) {
  switch (pl.f->dtype) {
    case LIRPA_F32: return grads_of_size<Split>(t, size, st);
    case LIRPA_BF16: return grads_of_size<bf16>(t, size, st);
    default: return grads_of_size<f16>(t, size, st);
  }
}

template <bool AKS, bool BKS, int EPI>
int run_tile(const FfnPlan& pl, const char* name, TileArgs& t, const Cut& cut, void* part,
             Joins* joins, hipStream_t st) {
  auto typed = [&](auto keep) {
    constexpr int K = decltype(keep)::value;
    switch (pl.f->dtype) {
      case LIRPA_F32: return tile_of_size<Split, AKS, BKS, EPI, K>(name, t, cut, (char*)part, joins, st);
      case LIRPA_BF16: return tile_of_size<bf16, AKS, BKS, EPI, K>(name, t, cut, (char*)part, joins, st);
      default: return tile_of_size<f16, AKS, BKS, EPI, K>(name, t, cut, (char*)part, joins, st);
    }
  };
  if constexpr (EPI == EPI_BACK)
    if (t.keep == LIRPA_KEEP_8) return typed(std::integral_constant<int, 8>{});
  return typed(std::integral_constant<int, 0>{});
}

// Up to kFewest tokens k_ffn_few is the faster one (us in bf16, against the tile kernel: 4096 x
// 10944, 1 token 59 and 66, 4 tokens 65 and 70, 8 the same; 1024 x 2752, 8 tokens 16 and 20).
// Weights that the tile kernel cannot read in place it reads up to kFewRows, rather than that they
// are copied.
constexpr int kFewest = 8, kFewRows = 64;

template <typename T, bool GATE, int TJ, int WAVES, int UN>
int few_product(const char* name, const FewArgs& a, hipStream_t st) {
  return launch_k(name, st, [&] {
    const unsigned blocks = (a.I + 15) / 16;
    if constexpr (sizeof(T) == 2) {
      // Rows off 4 bytes are read by words; the tokens' rows decide where a step has more of them
      // than of weights.  bf16, us, words / elements: 11 tokens, 3167 x 9543, 94 / 130, 50, 2047 x
      // 5501, 72 / 130.  Tokens alone off 4 bytes, 2046 x 5502: 50 of them 61 / 69, 10 33 / 29.
      const bool weights = (uintptr_t)a.A % 4 || a.lda % 2 ||
                           (GATE && ((uintptr_t)a.A2 % 4 || a.lda2 % 2));
      const bool words = weights || (TJ > 1 && ((uintptr_t)a.B % 4 || a.ldb % 2));
      if (words) {
        k_ffn_few<T, GATE, TJ, WAVES, UN, true><<<blocks, WAVES * 64, 0, st>>>(a);
        return;
      }
    }
    k_ffn_few<T, GATE, TJ, WAVES, UN, false><<<blocks, WAVES * 64, 0, st>>>(a);
  });
}

// GATE: waves a block of the gate product (16 of the down product); UN: steps in flight.
template <typename T, int TJ, int GATE, int UN>
int few_forward(const lirpa_ffn* f, int64_t rows, const void* x, int64_t ldx, void* out,
                int64_t ldo, void* hidden, hipStream_t st) {
  FewArgs a{};
  a.A = f->Wg;
  a.A2 = f->Wu;
  a.lda = f->ldg;
  a.lda2 = f->ldu;
  a.B = x;
  a.ldb = ldx;
  a.I = f->n_hidden;
  a.J = (int)rows;
  a.K = f->n_model;
  a.gate = f->gate;
  a.out = hidden;
  a.ldo = f->n_hidden;
  TRY((few_product<T, true, TJ, GATE, UN>("ffn_few_gate", a, st)));
  a.A = f->Wd;
  a.lda = f->ldd;
  a.B = hidden;
  a.ldb = f->n_hidden;
  a.I = f->n_model;
  a.K = f->n_hidden;
  a.out = out;
  a.ldo = ldo;
  return few_product<T, false, TJ, 16, UN>("ffn_few_down", a, st);
}

struct ForwardRoom {
  Operand x, wg, wu, wd, a;
  Cut cut_gate, cut_down;
  void* part;
  size_t bytes;
};
TileProblem gate_problem(const FfnPlan& pl, const ForwardRoom& r) {
  TileProblem p = problem(pl.F, pl.rows, pl.Dp, pl.Dp);
  add_segs(pl, p, r.wg, r.x);
  return p;
}
TileProblem down_problem(const FfnPlan& pl, const ForwardRoom& r) {
  TileProblem p = problem(pl.D, pl.rows, pl.Fp, pl.Fp);
  add_segs(pl, p, r.wd, r.a);
  return p;
}
ForwardRoom forward_room(FfnPlan& pl) {
  ForwardRoom r;
  r.x = pl.own(pl.rows, pl.D);
  if (!pl.in_in_place()) r.wg = pl.own(pl.F, pl.D), r.wu = pl.own(pl.F, pl.D);
  if (!pl.down_in_place()) r.wd = pl.own(pl.D, pl.F);
  r.a = pl.own(pl.rows, pl.F);
  const TileProblem gate = gate_problem(pl, r), down = down_problem(pl, r);
  const size_t gate_room = most_part_room(pl, &gate, 1, 2), down_room = most_part_room(pl, &down, 1);
  r.cut_gate = cut_of(&gate, 1, EPI_GATE, true, true, gate_room);
  r.cut_down = cut_of(&down, 1, EPI_STORE, true, true, down_room);
  // the gate product's sums are added before the down product's are written
  r.part = pl.ws.take(std::max(gate_room, down_room));
  r.bytes = pl.ws.at;
  return r;
}

int ffn_forward(const lirpa_ffn* f, int64_t rows, const void* x, int64_t ldx, void* out,
                int64_t ldo, int keep, void* g, void* u, void* ws, hipStream_t st) {
  FfnPlan pl(f, rows, ws);
  const bool in = pl.in_in_place(), down = pl.down_in_place();
  if (keep == LIRPA_KEEP_NONE && rows <= (in && down ? kFewest : kFewRows))
    return by_type(f->dtype, [&](auto t) {
      using T = decltype(t);
      // Large weights keep the memory busy with more on the way, small ones are done sooner with
      // fewer steps.  1 token, us with gate waves x steps in flight 8 x 2 / 8 x 4 / 16 x 4: 4096 x
      // 10944 bf16 58.5 / - / 57.1, float 123 / 108 / 109; 1024 x 2752 bf16 10.4 / 11.2 / 13.6,
      // float 18.2 / 19.4 / 23.0; 512 x 4400 float 17.9 / 23.1 / 27.8.  Gate product of 62 tokens,
      // 2816 x 616 float, 4 / 8 waves 52 / 44, of 64, 1024 x 2752, 24.5 / 21.6; 20 tokens, 8 / 16
      // waves, 25 / 27.
      constexpr int kLargeGate = sizeof(T) == 2 ? 16 : 8;
      const bool large = 3 * pl.D * pl.F * (int64_t)sizeof(T) >= (int64_t)64 << 20;
      if (rows <= 16 && large)
        return few_forward<T, 1, kLargeGate, 4>(f, rows, x, ldx, out, ldo, ws, st);
      if (rows <= 16) return few_forward<T, 1, 8, 2>(f, rows, x, ldx, out, ldo, ws, st);
      if (rows <= 32) return few_forward<T, 2, 8, 2>(f, rows, x, ldx, out, ldo, ws, st);
      return few_forward<T, 4, 8, 2>(f, rows, x, ldx, out, ldo, ws, st);
    });
  ForwardRoom r = forward_room(pl);
  Copies copies;
  copies.add(pl.in_place(x, ldx, pl.D), x, ldx, rows, pl.D, r.x);
  copies.add(in, f->Wg, f->ldg, pl.F, pl.D, r.wg);
  copies.add(in, f->Wu, f->ldu, pl.F, pl.D, r.wu);
  copies.add(down, f->Wd, f->ldd, pl.D, pl.F, r.wd);
  TRY(copies.run(pl, st));

  TileArgs t = tile_args(pl, keep);
  TileProblem& p = t.prob[0];
  p = gate_problem(pl, r);
  for (int s = 0; s < p.nseg; ++s) t.A2[s] = r.wu.p + (p.A[s] - r.wg.p);
  p.out = (void*)r.a.p;
  p.ldo = r.a.ld;
  p.pad_i = (int)pl.Fp;
  p.plane = r.a.plane;
  t.g = g;
  t.u = u;
  t.ge = (uint8_t*)g + q8_exps_at(rows, (int)pl.F);
  t.ue = (uint8_t*)u + q8_exps_at(rows, (int)pl.F);
  TRY((run_tile<false, false, EPI_GATE>(pl, "ffn_gate_up", t, r.cut_gate, r.part, nullptr,
                                          st)));

  Joins joins;
  t = tile_args(pl, LIRPA_KEEP_NONE);
  t.prob[0] = down_problem(pl, r);
  t.prob[0].out = out;
  t.prob[0].ldo = ldo;
  TRY((run_tile<false, false, EPI_STORE>(pl, "ffn_down", t, r.cut_down, r.part, &joins, st)));
  return joins.run(pl, st);
}

struct BackwardRoom {
  Operand dout, x, wg, wu, wd, a, dg, du;
  Cut cut_gate, cut_grads;
  void* part;
  size_t bytes;
};
TileProblem da_problem(const FfnPlan& pl, const BackwardRoom& r) {
  TileProblem p = problem(pl.F, pl.rows, pl.D, pl.Dp);
  add_segs(pl, p, r.wd, r.dout);
  return p;
}
// dx, dWg, dWu and dWd.
void grad_problems(const FfnPlan& pl, const BackwardRoom& r, bool packed_x, TileProblem* p) {
  p[0] = problem(pl.D, pl.rows, pl.F, pl.Fp);
  add_segs(pl, p[0], r.wg, r.dg);
  add_segs(pl, p[0], r.wu, r.du);
  p[1] = p[2] = problem(pl.D, pl.F, pl.rows, pl.rows);
  add_segs(pl, p[1], r.x, r.dg, packed_x);
  add_segs(pl, p[2], r.x, r.du, packed_x);
  p[3] = problem(pl.F, pl.D, pl.rows, pl.rows);
  add_segs(pl, p[3], r.a, r.dout);
  for (int i = 1; i < 4; ++i) p[i].b_strided = true;
}
BackwardRoom backward_room(FfnPlan& pl, bool packed_x) {
  BackwardRoom r;
  r.dout = pl.own(pl.rows, pl.D);
  r.x = pl.own(pl.rows, pl.D);
  if (!pl.in_in_place()) r.wg = pl.own(pl.F, pl.D), r.wu = pl.own(pl.F, pl.D);
  if (!pl.down_in_place()) r.wd = pl.own(pl.D, pl.F);
  r.a = pl.own(pl.rows, pl.F);
  r.dg = pl.own(pl.rows, pl.F);
  r.du = pl.own(pl.rows, pl.F);
  const TileProblem da = da_problem(pl, r);
  // cut as if all four were wanted: a gradient does not depend on which others are
  TileProblem grads[4];
  grad_problems(pl, r, packed_x, grads);
  const size_t da_room = most_part_room(pl, &da, 1), grads_room = most_part_room(pl, grads, 4);
  r.cut_gate = cut_of(&da, 1, EPI_BACK, !pl.f32, false, da_room);
  r.cut_grads = cut_of(grads, 4, EPI_STORE, true, false, grads_room);
  r.part = pl.ws.take(std::max(da_room, grads_room));  // da's sums are added first
  r.bytes = pl.ws.at;
  return r;
}

int ffn_backward(const lirpa_ffn* f, int64_t rows, const void* dout, int64_t lddo, int keep,
                 const void* x, int64_t ldx, const void* g, const void* u, void* dx, int64_t lddx,
                 void* dWg, void* dWu, void* dWd, void* ws, hipStream_t st) {
  FfnPlan pl(f, rows, ws);
  const bool packed = keep == LIRPA_KEEP_8;
  BackwardRoom r = backward_room(pl, packed);
  Copies copies;
  copies.add(pl.in_place(dout, lddo, pl.D), dout, lddo, rows, pl.D, r.dout);
  if (dx) {
    copies.add(pl.in_in_place(), f->Wg, f->ldg, pl.F, pl.D, r.wg);
    copies.add(pl.in_in_place(), f->Wu, f->ldu, pl.F, pl.D, r.wu);
  }
  copies.add(pl.down_in_place(), f->Wd, f->ldd, pl.D, pl.F, r.wd);
  if (dWg || dWu) {
    if (packed)
      copies.add_packed(x, rows, pl.D, r.x);
    else
      copies.add(pl.in_place(x, ldx, pl.D), x, ldx, rows, pl.D, r.x);
  }
  TRY(copies.run(pl, st));

  // act(g) u, dg and du
  TileArgs t = tile_args(pl, keep);
  TileProblem& p = t.prob[0];
  p = da_problem(pl, r);
  p.out = dWd ? (void*)r.a.p : nullptr;
  p.ldo = r.a.ld;
  p.plane = r.a.plane;
  p.pad_i = (int)pl.Fp;
  t.dg = dx || dWg ? (void*)r.dg.p : nullptr;
  t.du = dx || dWu ? (void*)r.du.p : nullptr;
  t.g = (void*)g;
  t.u = (void*)u;
  t.ge = (uint8_t*)g + q8_exps_at(rows, (int)pl.F);
  t.ue = (uint8_t*)u + q8_exps_at(rows, (int)pl.F);
  TRY((run_tile<true, false, EPI_BACK>(pl, "ffn_back_gate", t, r.cut_gate, r.part, nullptr,
                                         st)));

  Joins joins;
  t = tile_args(pl, LIRPA_KEEP_NONE);
  t.count = 0;
  TileProblem grads[4];
  grad_problems(pl, r, packed, grads);
  void* outs[4] = {dx, dWg, dWu, dWd};
  const int64_t lds[4] = {lddx, pl.D, pl.D, pl.F};
  char* part = (char*)r.part;
  for (int i = 0; i < 4; ++i) {
    if (!outs[i]) continue;
    TileProblem& q = t.prob[t.count++];
    q = grads[i];
    q.out = outs[i];
    q.ldo = lds[i];
    split(q, r.cut_grads.splits[i], part);
    if (q.splits > 1) joins.add(q);
  }
  TRY(run_grads(pl, t, r.cut_grads.size, st));
  return joins.run(pl, st);
}

size_t ffn_bytes(const lirpa_ffn* f, int64_t rows, bool backward) {
  if (!backward) {
    FfnPlan pl(f, rows, nullptr);
    return forward_room(pl).bytes;
  }
  FfnPlan full(f, rows, nullptr), packed(f, rows, nullptr);
  return std::max(backward_room(full, false).bytes, backward_room(packed, true).bytes);
}

}  // namespace

extern "C" {

size_t lirpa_q8_bytes(int64_t rows, int n) {
  if (rows < 0 || rows > kMaxRows || n < 1 || n > kMaxWidth) return 0;
  return q8_bytes(rows, n);
}

int lirpa_q8_pack(int dtype, int64_t rows, int n, const void* x, int64_t ldx, void* q8,
                  hipStream_t stream) {
  return guarded([&] {
    TRY(check_shape("lirpa_q8_pack", dtype, rows, n));
    if (rows == 0) return (int)LIRPA_OK;
    TRY(check_rows("lirpa_q8_pack", "x", dtype, x, ldx, n));
    TRY(check_q8("lirpa_q8_pack", "q8", q8));
    return by_type(dtype, [&](auto t) {
      return q8_pack(rows, n, (const decltype(t)*)x, ldx, q8, stream);
    });
  });
}

int lirpa_q8_unpack(int dtype, int64_t rows, int n, const void* q8, void* x, int64_t ldx,
                    hipStream_t stream) {
  return guarded([&] {
    TRY(check_shape("lirpa_q8_unpack", dtype, rows, n));
    if (rows == 0) return (int)LIRPA_OK;
    TRY(check_rows("lirpa_q8_unpack", "x", dtype, x, ldx, n));
    TRY(check_q8("lirpa_q8_unpack", "q8", q8));
    return by_type(dtype, [&](auto t) {
      return q8_unpack(rows, n, q8, (decltype(t)*)x, ldx, stream);
    });
  });
}

int lirpa_norm_forward(int dtype, int64_t rows, int n, const void* x, int64_t ldx,
                       const void* res, int64_t ldr, const void* w, float eps, void* sum,
                       int64_t lds, void* y, int64_t ldy, void* y8, float* rstd,
                       hipStream_t stream) {
  return guarded([&] {
    const char* who = "lirpa_norm_forward";
    TRY(check_shape(who, dtype, rows, n));
    if (!(eps >= 0.f) || !std::isfinite(eps))
      return fail(LIRPA_EINVAL, "%s: eps must be finite and >= 0", who);
    if (rows == 0) return (int)LIRPA_OK;  // an empty buffer may be null
    if (!sum && !y && !y8 && !rstd) return fail(LIRPA_EINVAL, "%s: no output is wanted", who);
    TRY(check_rows(who, "x", dtype, x, ldx, n));
    if (res) TRY(check_rows(who, "res", dtype, res, ldr, n));
    TRY(check_rows(who, "w", dtype, w, n, n));
    if (sum) TRY(check_rows(who, "sum", dtype, sum, lds, n));
    if (y) TRY(check_rows(who, "y", dtype, y, ldy, n));
    if (y8) TRY(check_q8(who, "y8", y8));
    TRY(check_in_place(who, "sum", sum, lds, "x", x, ldx, rows));
    TRY(check_in_place(who, "sum", sum, lds, "res", res, ldr, rows));
    return by_type(dtype, [&](auto t) {
      using T = decltype(t);
      NormFwd<T> a{};
      a.x = (const T*)x;
      a.res = (const T*)res;
      a.w = (const T*)w;
      a.ldx = ldx;
      a.ldr = ldr;
      a.lds = lds;
      a.ldy = ldy;
      a.rows = rows;
      a.n = n;
      a.eps = eps;
      a.sum = (T*)sum;
      a.y = (T*)y;
      a.q = (int8_t*)y8;
      a.exps = y8 ? (uint8_t*)y8 + q8_exps_at(rows, n) : nullptr;
      a.rstd = rstd;
      return norm_fwd(a, stream);
    });
  });
}

size_t lirpa_norm_workspace_bytes(int64_t rows, int n) {
  if (rows < 0 || rows > kMaxRows || n < 1 || n > kMaxWidth) return 0;
  return std::max<size_t>(256, (size_t)norm_bwd_blocks(rows, n) * n * sizeof(float));
}

int lirpa_norm_backward(int dtype, int64_t rows, int n, const void* dy, int64_t lddy,
                        const void* dsum, int64_t ldds, const void* h, int64_t ldh,
                        const void* w, const float* rstd, void* dh, int64_t lddh, void* dw,
                        void* ws, size_t ws_bytes, hipStream_t stream) {
  return guarded([&] {
    const char* who = "lirpa_norm_backward";
    TRY(check_shape(who, dtype, rows, n));
    if (!dh && !dw && rows > 0) return fail(LIRPA_EINVAL, "%s: no output is wanted", who);
    if (rows > 0) {
      TRY(check_rows(who, "dy", dtype, dy, lddy, n));
      if (dsum) TRY(check_rows(who, "dsum", dtype, dsum, ldds, n));
      TRY(check_rows(who, "h", dtype, h, ldh, n));
      TRY(check_rows(who, "w", dtype, w, n, n));
      if (!rstd) return fail(LIRPA_EINVAL, "%s: rstd is null", who);
      if (dh) TRY(check_rows(who, "dh", dtype, dh, lddh, n));
      TRY(check_in_place(who, "dh", dh, lddh, "dy", dy, lddy, rows));
      TRY(check_in_place(who, "dh", dh, lddh, "dsum", dsum, ldds, rows));
    }
    if (dw) {
      TRY(check_rows(who, "dw", dtype, dw, n, n));
      if (!ws) return fail(LIRPA_EINVAL, "%s: the workspace is null", who);
      if (!aligned16(ws))
        return fail(LIRPA_EINVAL, "%s: the workspace does not start on 16 bytes", who);
      const size_t need = lirpa_norm_workspace_bytes(rows, n);
      if (ws_bytes < need)
        return fail(LIRPA_ENOMEM, "%s: the workspace has %zu bytes, %zu are needed", who, ws_bytes,
                    need);
    }
    return by_type(dtype, [&](auto t) {
      using T = decltype(t);
      NormBwd<T> a{};
      a.dy = (const T*)dy;
      a.dsum = (const T*)dsum;
      a.h = (const T*)h;
      a.w = (const T*)w;
      a.lddy = lddy;
      a.ldds = ldds;
      a.ldh = ldh;
      a.lddh = lddh;
      a.rows = rows;
      a.n = n;
      a.rstd = rstd;
      a.dh = (T*)dh;
      return norm_bwd(a, (T*)dw, (float*)ws, stream);
    });
  });
}

size_t lirpa_ffn_workspace_bytes(const lirpa_ffn* ffn, int64_t rows, int backward) {
  if (check_ffn("lirpa_ffn_workspace_bytes", ffn) != LIRPA_OK) return 0;
  if (rows < 0 || rows > kMaxRows || (backward != 0 && backward != 1)) {
    fail(LIRPA_EINVAL, "lirpa_ffn_workspace_bytes: rows or backward out of range");
    return 0;
  }
  return std::max<size_t>(256, ffn_bytes(ffn, rows, backward == 1));
}

int lirpa_ffn_forward(const lirpa_ffn* ffn, int64_t rows, const void* x, int64_t ldx, void* out,
                      int64_t ldo, int keep, void* g, void* u, void* ws, size_t ws_bytes,
                      hipStream_t stream) {
  return guarded([&] {
    const char* who = "lirpa_ffn_forward";
    TRY(check_ffn(who, ffn));
    TRY(check_shape(who, ffn->dtype, rows, ffn->n_model));
    if (keep != LIRPA_KEEP_NONE && keep != LIRPA_KEEP_FULL && keep != LIRPA_KEEP_8)
      return fail(LIRPA_EINVAL, "%s: keep %d is none of lirpa_keep", who, keep);
    if (keep == LIRPA_KEEP_NONE && (g || u))
      return fail(LIRPA_EINVAL, "%s: g and u are null where nothing is kept", who);
    if (rows == 0) return (int)LIRPA_OK;
    TRY(check_rows(who, "x", ffn->dtype, x, ldx, ffn->n_model));
    TRY(check_rows(who, "out", ffn->dtype, out, ldo, ffn->n_model));
    if (keep == LIRPA_KEEP_8) {
      TRY(check_q8(who, "g", g));
      TRY(check_q8(who, "u", u));
    } else if (keep == LIRPA_KEEP_FULL) {
      TRY(check_rows(who, "g", ffn->dtype, g, ffn->n_hidden, ffn->n_hidden));
      TRY(check_rows(who, "u", ffn->dtype, u, ffn->n_hidden, ffn->n_hidden));
    }
    if (!ws) return fail(LIRPA_EINVAL, "%s: the workspace is null", who);
    if (!aligned16(ws))
      return fail(LIRPA_EINVAL, "%s: the workspace does not start on 16 bytes", who);
    const size_t need = lirpa_ffn_workspace_bytes(ffn, rows, 0);
    if (ws_bytes < need)
      return fail(LIRPA_ENOMEM, "%s: the workspace has %zu bytes, %zu are needed", who, ws_bytes,
                  need);
    return ffn_forward(ffn, rows, x, ldx, out, ldo, keep, g, u, ws, stream);
  });
}

int lirpa_ffn_backward(const lirpa_ffn* ffn, int64_t rows, const void* dout, int64_t lddo,
                       int keep, const void* x, int64_t ldx, const void* g, const void* u,
                       void* dx, int64_t lddx, void* dWg, void* dWu, void* dWd, void* ws,
                       size_t ws_bytes, hipStream_t stream) {
  return guarded([&] {
    const char* who = "lirpa_ffn_backward";
    TRY(check_ffn(who, ffn));
    const int t = ffn->dtype, D = ffn->n_model, F = ffn->n_hidden;
    TRY(check_shape(who, t, rows, D));
    if (keep != LIRPA_KEEP_FULL && keep != LIRPA_KEEP_8)
      return fail(LIRPA_EINVAL, "%s: keep must be LIRPA_KEEP_FULL or LIRPA_KEEP_8", who);
    if (!dx && !dWg && !dWu && !dWd && rows > 0)
      return fail(LIRPA_EINVAL, "%s: no output is wanted", who);
    if (rows > 0) {
      TRY(check_rows(who, "dout", t, dout, lddo, D));
      if (keep == LIRPA_KEEP_8) {
        if (dWg || dWu) TRY(check_q8(who, "x", x));
        TRY(check_q8(who, "g", g));
        TRY(check_q8(who, "u", u));
      } else {
        if (dWg || dWu) TRY(check_rows(who, "x", t, x, ldx, D));
        TRY(check_rows(who, "g", t, g, F, F));
        TRY(check_rows(who, "u", t, u, F, F));
      }
      if (dx) TRY(check_rows(who, "dx", t, dx, lddx, D));
    }
    if (dWg) TRY(check_rows(who, "dWg", t, dWg, D, D));
    if (dWu) TRY(check_rows(who, "dWu", t, dWu, D, D));
    if (dWd) TRY(check_rows(who, "dWd", t, dWd, F, F));
    if (!ws) return fail(LIRPA_EINVAL, "%s: the workspace is null", who);
    if (!aligned16(ws))
      return fail(LIRPA_EINVAL, "%s: the workspace does not start on 16 bytes", who);
    const size_t need = lirpa_ffn_workspace_bytes(ffn, rows, 1);
    if (ws_bytes < need)
      return fail(LIRPA_ENOMEM, "%s: the workspace has %zu bytes, %zu are needed", who, ws_bytes,
                  need);
    return ffn_backward(ffn, rows, dout, lddo, keep, x, ldx, g, u, dx, lddx, dWg, dWu, dWd, ws,
                        stream);
  });
}

}  // extern "C"
