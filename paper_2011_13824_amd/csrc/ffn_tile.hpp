// Matrix products of the gated feed-forward block on 16-bit matrix instructions.
//
//   C[j][i] = sum over segments s and k of A_s(i, k) * B_s(j, k),  32-bit sums
//   out = (act(x Wg^T) * (x Wu^T)) Wd^T
//   da = dout Wd, dg = da u act'(g), du = da act(g)
//   dx = dg Wg + du Wu, dWg = dg^T x, dWu = du^T x, dWd = dout^T (act(g) u)
//
// i runs over the contiguous dimension of the output (features), j over its rows (tokens).  An
// operand is stored k-contiguous ([i][k]) or k-strided ([k][i]); the second kind is transposed on
// its way from LDS into registers (ds_read_tr16_b64), so no product needs a transposed copy.  The
// same kernel does every product of the block:
//
//   gate and up   A = Wg | Wu (k-contiguous)     B = x (k-contiguous)      EPI_GATE
//   down          A = Wd (k-contiguous)          B = act(g) u              EPI_STORE
//   da            A = Wd (k-strided)             B = dout                  EPI_BACK
//   dx            A = Wg, Wu (k-strided)         B = dg, du                EPI_STORE, two segments
//   dWg, dWu      A = x (k-strided)              B = dg, du (k-strided)    EPI_STORE, one launch
//   dWd           A = act(g) u (k-strided)       B = dout (k-strided)      EPI_STORE, with them
//
// 32-bit operands are three bf16 parts (hi + mid + lo = 24 bits, from magnitudes of 2^-109 on: parts
// under bf16's least normal number may be lost); a product is then six segments,
// those of the largest parts, smallest first, and the error stays that of a 32-bit sum (6e-7 of
// the result's norm against 64 bits, where a library's 32-bit product has 1.3e-6).  Their rate
// counts a sixth: six bf16 products at 1.2 PFLOP/s, where the 32-bit matrix instruction ends at
// 157 TFLOP/s.
//
// act(g) u, dg and du are rounded to the tensors' type between two products: they are operands of
// 16-bit instructions.  That is one more rounding of up to 2^-8 (bf16) or 2^-11 (f16) of every term,
// of random sign: a bf16 result is off by 0.0023 of its norm, where operands of 32 bits leave
// 0.0017.
//
// How the loop is fed (8192^3 in bf16 on one MI355X, TFLOP/s; the matrix instructions alone reach
// 1640 to 1930 there, a third less with random operands than with zeros, for power):
//  - Two stages of 64 k, copied into LDS at once, fragments read when needed: 1109 (both operands
//    k-contiguous), 1028 (both k-strided).
//  - Copies go from memory straight into LDS.  Rows of 64 bytes a copy reach 17 to 22 TB/s over the
//    chip, rows of 128 bytes and more 32 to 34: a tile is 64 k, 128 bytes of a row.
//  - A copy that finds the address unit busy holds back everything its wave issues after it, so a
//    burst of copies stops the matrix instructions.  They are issued one by one between them.
//  - Fragments are read half a tile ahead into registers of their own, and a barrier a tile is
//    left.  LDS holds five units (a tile of one operand each), A and B in turn, so that copies are
//    one to one and a half tiles ahead: 1264 and 1366.
//  - 8 waves of 128 x 64 rather than 4 of 128 x 128, which read a third less from LDS: two waves a
//    SIMD hide each other's waits, and four waves' sums do not fit beside their fragments without
//    moves (988 as built by the compiler).
// A large library product reaches 1400 to 1445 with k-contiguous operands, 1088 to 1170 with
// k-strided ones.
#pragma once

#include <type_traits>

#include "lm_types.hpp"

namespace lm {

enum Epi { EPI_STORE, EPI_GATE, EPI_BACK };
enum Gate { RELU = 0, SILU = 1, GELU = 2 };

constexpr int kMaxSegs = 12;
constexpr int kBK = 64;  // k a tile: 128 bytes of a k-contiguous row, the width of a cache line
constexpr int kMaxProblems = 4;

// One product.
struct TileProblem {
  const char* A[kMaxSegs];
  const char* B[kMaxSegs];
  int64_t lda, ldb;    // bytes between rows, the same for all segments
  int nseg;
  int KA, KB;          // k extents (equal up to the zero padding of a packed operand)
  bool b_strided;      // gradients: B is k-strided too
  int I, J;            // output sizes
  int tiles_i, tiles_j;
  unsigned first;      // block of its first tile
  int splits;          // blocks that share a tile's k; over 1, their sums go to
  float* part;         // part[split][J][part_ld] (EPI_GATE: [split][2][J][part_ld], g and u) and
                       // are added by k_ffn_join or k_ffn_finish
  int64_t part_ld;
  void* out;           // the tensors' type (EPI_STORE), else an operand of a later product
  int64_t ldo;         // elements
  int pad_i;           // columns [I, pad_i) of an operand are written as 0
  int64_t plane;       // elements between the parts of a 32-bit operand
};

// A launch: products that do not depend on one another (EPI_STORE), or one with its epilogue.
struct TileArgs {
  TileProblem prob[kMaxProblems];
  int count;
  const char* A2[kMaxSegs];  // EPI_GATE: the rows of Wu, as those of Wg
  int gate, keep;            // keep: -1, 0, 8
  void *g, *u;               // what is kept: [J][I] or packed
  uint8_t *ge, *ue;          // exponents of the packed form
  void *dg, *du;             // EPI_BACK
};

__device__ __forceinline__ int up32(int n) { return (n + 31) & ~31; }

__device__ __forceinline__ void read8(const float* p, float (&x)[8]) {
  const f32x4 lo = *(const f32x4*)p, hi = *(const f32x4*)(p + 4);
#pragma unroll
  for (int r = 0; r < 4; ++r) x[r] = lo[r], x[4 + r] = hi[r];
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

// Operands of the tile kernel: bf16, f16, or three bf16 parts of a float (Split).
struct Split {};

// The next bf16 part of v, which keeps what is left.  The first part of a finite v over bf16's
// largest is that, and the second holds the rest; an infinity or a NaN is its first part alone.
__device__ __forceinline__ float take_part(float& v, bool first) {
  constexpr float kMost = 3.38953139e38f;  // 255 * 2^120
  const float whole = v;
  float p = (float)(bf16)(first ? __builtin_amdgcn_fmed3f(v, -kMost, kMost) : v);
  v -= p;
  if (first && !(fabsf(v) < INFINITY)) p = whole, v = 0.f;
  return p;
}

template <typename T>
struct Kind {
  using Half = T;  // what the matrix instruction takes
  using Whole = T; // the tensors' type
  static constexpr int kParts = 1;
};
template <>
struct Kind<Split> {
  using Half = bf16;
  using Whole = float;
  static constexpr int kParts = 3;
};

template <typename T>
struct Mfma;
template <>
struct Mfma<bf16> {
  typedef bf16 x8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 mac(x8 a, x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ void add(s16x8 a, s16x8 b, f32x4& c) {
    c = mac(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c);
  }
};
template <>
struct Mfma<f16> {
  typedef f16 x8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 mac(x8 a, x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ void add(s16x8 a, s16x8 b, f32x4& c) {
    c = mac(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c);
  }
};

// act(x) and act'(x).  `fast`: e^x and the reciprocal with the hardware's own instructions, 1e-6
// off near 0 and x^2 2^-24 further out, far under the rounding of a 16-bit type.
//
// Phi(x) for x <= 0 is erfc(z) / 2 with z = |x| / sqrt(2), and erfc(z) e^(z^2) is t P(t) with
// t = 1 / (1 + 0.4 z): P is a fit of degree 8 in the relative error (1.3e-7 over t in (0, 1]), made
// for this file by reweighted least squares.  e^(-z^2) is the slope's too.
__device__ __forceinline__ void gate_fn(int gate, bool fast, float x, float& act, float& slope) {
  if (gate == RELU) {
    act = fmaxf(x, 0.f);
    slope = x > 0.f ? 1.f : 0.f;
    if (x != x) act = slope = x;
  } else if (gate == SILU) {
    const float p = fast ? __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950409f * x))
                         : 1.f / (1.f + expf(-x));
    act = x * p;
    slope = p * (1.f + x * (1.f - p));
  } else {
    const float below = 1.f + 0.28284271247f * fabsf(x), xx = x * x;
    const float t = fast ? __builtin_amdgcn_rcpf(below) : 1.f / below;
    float e;
    if (fast) {
      e = __builtin_amdgcn_exp2f(-0.72134752044f * xx);
    } else {  // what the square's rounding leaves would be multiplied by the square
      const float rest = xx < 1e30f ? fmaf(x, x, -xx) : 0.f;
      e = expf(-0.5f * xx) * (1.f - 0.5f * rest);
    }
    float p = 0.050272651f;
    p = fmaf(p, t, -0.182943851f);
    p = fmaf(p, t, 0.169155225f);
    p = fmaf(p, t, -0.00566805014f);
    p = fmaf(p, t, 0.141461045f);
    p = fmaf(p, t, 0.168533847f);
    p = fmaf(p, t, 0.20784387f);
    p = fmaf(p, t, 0.225669518f);
    p = fmaf(p, t, 0.225675866f);
    p *= 0.5f * t * e;
    if (x > 0.f) p = 1.f - p;
    act = x * p;
    slope = p + x * (0.39894228040143268f * e);
  }
}

// 16 bytes from global memory straight into LDS, lane l's at `lds` + 16 l (`lds` is uniform).  An
// offset of kOutside is past the descriptor's end, and brings zeros.  The compiler does not see
// these as loads: wait_all() stands between them and the reads.
constexpr uint32_t kOutside = 0x80000000u;
constexpr uint32_t kExtent = 0x7fffffffu;

__device__ __forceinline__ u32x4 descriptor(const char* p, uint32_t bytes) {
  const uint64_t a = (uint64_t)p;
  u32x4 d;
  d[0] = (uint32_t)a;
  d[1] = (uint32_t)(a >> 32) & 0xffffu;
  d[2] = bytes;
  d[3] = 0x00020000u;
  return d;
}
__device__ __forceinline__ void bring16(u32x4 desc, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds),
               "v"(offset), "s"(desc)
               : "memory", "m0");
}
__device__ __forceinline__ void wait_all() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
// All but the newest N of this thread's copies have arrived, and then every thread's.
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"(N) : "memory");
}

typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) s16x8 lds_s16x8;

// Where an operand's tile (R rows of i or j, kBK of k) lies in LDS.
//   k-contiguous: row r is 8 pieces of 16 bytes, piece p at p ^ (r / 2 % 8): the 16 rows that one
//   read takes then start in 16 different 16-byte columns of the 256 bytes of banks (without it a
//   read takes 4 cycles more).
//   k-strided: line k is R / 8 pieces, piece p at p ^ 2 f(k), f(k) = k % 4 + 4 (k / 8 % 2): a
//   transposing read takes 32 bytes of 4 lines, from 2 groups of lanes at k and k + 8.  Two lines
//   of 8 pieces fill the banks, and f(k) = k / 2 % 2 + 2 (k / 8 % 2) does.
template <bool KS, int R>
struct Lay {
  static constexpr int kPieces = KS ? R / 8 : kBK / 8;  // of a line
  static constexpr int kBytes = R * kBK * 2;
  static __device__ __forceinline__ int swizzle(int line) {
    if (!KS) return (line >> 1) & 7;
    if (R == 64) return (((line >> 1) & 1) | ((line >> 3) & 1) << 1) << 1;
    return ((line & 3) | ((line >> 3) & 1) << 2) << 1;
  }
};

// One operand's copies: thread t of THREADS brings pieces t, t + THREADS, ... of a tile.  Copy r
// lies kLines lines after copy 0, at the same place of its line.
template <bool KS, int R, int THREADS>
struct Bringer {
  using L = Lay<KS, R>;
  static constexpr int kLoads = L::kBytes / 16 / THREADS;
  static constexpr int kLines = THREADS / L::kPieces;
  static_assert(kLines % 16 == 0, "the swizzle repeats after 16 lines");
  uint32_t off;    // from the tile's corner; kOutside for columns past the end (k-strided)
  int k;           // first k of the piece (k-contiguous) or the line's k
  int64_t step;    // bytes of kLines lines
  uint32_t bytes;  // k-contiguous: of the rows that exist

  // `rows`: valid rows from the tile's corner on.
  __device__ __forceinline__ void init(int64_t ld, int rows) {
    const int line = threadIdx.x / L::kPieces;
    const int p = (threadIdx.x % L::kPieces) ^ L::swizzle(line);
    k = KS ? line : p * 8;
    off = !KS || p * 8 < rows ? (uint32_t)(line * ld) + p * 16 : kOutside;
    step = kLines * ld;
    bytes = __builtin_amdgcn_readfirstlane(
        KS ? kExtent : (uint32_t)min((int64_t)min(rows, R) * ld, (int64_t)kExtent));
  }
  // Copy r of the tile at `corner`, of which `left` k exist, none where it is <= 0.
  __device__ __forceinline__ void bring(const char* corner, int left, uint32_t lds, int r) const {
    const uint32_t skip = (uint32_t)(r * step);
    const uint32_t left_bytes = __builtin_amdgcn_readfirstlane(bytes > skip ? bytes - skip : 0);
    const u32x4 d = descriptor(corner + r * step, KS ? kExtent : left_bytes);
    bring16(d, k + (KS ? r * kLines : 0) < left ? off : kOutside, lds + r * THREADS * 16);
  }
};

// A fragment: 8 k of one row per lane (row = lane % 16, k = 8 (lane / 16) + 0..7 of 32).
template <bool KS, int R>
struct Reader {
  using L = Lay<KS, R>;
  uint32_t at;  // of fragment 0 of the first half of a tile at 0
  // `row0`: the wave's first row in the tile; fragments lie 16 rows apart.
  __device__ __forceinline__ void init(int row0) {
    const int lane = threadIdx.x & 63, m = lane & 15, q = lane >> 4;
    if constexpr (KS) {
      const int k = q * 8 + (m >> 2), p = row0 / 8 + ((m & 3) >> 1);
      at = k * R * 2 + (p ^ L::swizzle(k)) * 16 + (m & 1) * 8;
    } else {
      at = (row0 + m) * (kBK * 2) + (q ^ L::swizzle(m)) * 16;
    }
  }
  // Fragment f of half ks of the tile at `tile`.  The bits that the swizzle mixes are changed
  // with an exclusive or: pieces 2 f of up to 16 (k-strided), 4 ks of 8.
  __device__ __forceinline__ s16x8 read(uint32_t tile, int f, int ks) const {
    if constexpr (KS) {
      const uint32_t a = (tile + at) ^ (f * 32);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_s16x4*)(uintptr_t)(a + ks * 32 * R * 2));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_s16x4*)(uintptr_t)(a + (ks * 32 + 4) * R * 2));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      const uint32_t a = (tile + at) ^ (ks * 64);
      return *(lds_s16x8*)(uintptr_t)(a + f * (16 * kBK * 2));
    }
  }
};

// Where a lane's piece, eight consecutive features of a token, lies in the arrays of an epilogue:
// 32-bit offsets from the row that the wave has come to, whose address is uniform.
struct Piece8 {
  int col;          // of the first feature
  uint32_t token;   // rows from the wave's row on
  uint32_t q, e;    // bytes in a packed array and in its exponents
};

// An operand of a later product: 16 bits, or three bf16 parts of a 32-bit value.  The columns
// [I, pad_i) are cleared.
template <typename T>
__device__ __forceinline__ void put_operand(const TileProblem& p, void* base, int64_t row,
                                            const Piece8& l, const float (&v)[8]) {
  using H = typename Kind<T>::Half;
  char* to = (char*)base + row * p.ldo * sizeof(H);
  const uint32_t at = (l.token * (uint32_t)p.ldo + l.col) * sizeof(H);
  float rest[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) rest[r] = l.col + r < p.I ? v[r] : 0.f;
  if constexpr (Kind<T>::kParts == 1) {
    store_row<H, 8>((H*)(to + at), p.pad_i - l.col, rest);
  } else {
#pragma unroll
    for (int part = 0; part < 3; ++part) {
      float x[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) x[r] = take_part(rest[r], part == 0);
      store_row<H, 8>((H*)(to + part * p.plane * sizeof(H) + at), p.pad_i - l.col, x);
    }
  }
}

template <typename T>
__device__ __forceinline__ void put_output(const TileProblem& p, void* base, int64_t ld, int64_t row,
                                           const Piece8& l, const float (&v)[8]) {
  using W = typename Kind<T>::Whole;
  char* to = (char*)base + row * ld * sizeof(W);
  store_row<W, 8>((W*)(to + (l.token * (uint32_t)ld + l.col) * sizeof(W)), p.I - l.col, v);
}

// What the forward pass keeps: packed with a scale for 32 features (four neighbouring lanes), or
// as it is.  Every lane of the wave comes here.
template <typename T>
__device__ __forceinline__ void keep8(const TileProblem& p, int keep, void* base, uint8_t* exps, int64_t row,
                                      const Piece8& l, const float (&v)[8]) {
  const bool in = row + l.token < p.J && l.col < up32(p.I);
  if (keep != 8) {
    if (in) put_output<T>(p, base, p.I, row, l, v);
    return;
  }
  const int e = group_exponent4(v), groups = groups_of(p.I);
  if (!in) return;
  store_global((char*)base + row * groups * kGroup + l.q, pack8(v, e));
  if ((l.col & 31) == 0) store_global(exps + row * groups + l.e, (uint8_t)e);
}

// What was kept, loaded now and turned into values later.
template <typename T, int KEEP>
struct Kept8 {
  using W = typename Kind<T>::Whole;
  Vec<W, 8> raw;
  __device__ __forceinline__ void load(const TileProblem& p, const void* base, const uint8_t*,
                                       int64_t row, const Piece8& l) {
    if (row + l.token >= p.J || l.col >= p.I) return;
    const W* from = (const W*)((const char*)base + row * p.I * sizeof(W) +
                            (l.token * (uint32_t)p.I + l.col) * sizeof(W));
    if (p.I - l.col >= 8) {
      raw = load_global<Vec<W, 8>>(from);
    } else {
#pragma unroll
      for (int r = 0; r < 8; ++r) raw[r] = l.col + r < p.I ? load_global<W>(from + r) : (W)0.f;
    }
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
    for (int r = 0; r < 8; ++r) v[r] = (float)raw[r];
  }
};
template <typename T>
struct Kept8<T, 8> {
  u32x2 w;
  int e;
  __device__ __forceinline__ void load(const TileProblem& p, const void* base, const uint8_t* exps,
                                       int64_t row, const Piece8& l) {
    // no branch: what lies past the end is read from the array's start, and not used
    const int groups = groups_of(p.I);
    const bool in = row + l.token < p.J && l.col < p.I;
    const int64_t first = row < p.J ? row : 0;
    w = load_global<u32x2>((const char*)base + first * groups * kGroup + (in ? l.q : 0));
    e = load_global<uint8_t>(exps + first * groups + (in ? l.e : 0));
  }
  __device__ __forceinline__ void values(float (&v)[8]) const { unpack8(w, e, v); }
};

// The epilogues on eight consecutive features of a token.  Every lane of the wave comes here, `in`
// where its token exists.

// act(g) u and what is kept; x: g.
template <typename T>
__device__ __forceinline__ void finish_gate(const TileArgs& a, const TileProblem& p, int64_t row,
                                            const Piece8& at, bool in, float (&x)[8],
                                            float (&u)[8]) {
  if (a.keep >= 0) {
    keep8<T>(p, a.keep, a.g, a.ge, row, at, x);
    keep8<T>(p, a.keep, a.u, a.ue, row, at, u);
  }
  if (!in || at.col >= p.pad_i) return;
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    float act, slope;
    gate_fn(a.gate, Kind<T>::kParts == 1, x[r], act, slope);
    u[r] *= act;
  }
  put_operand<T>(p, p.out, row, at, u);
}

// act(g) u, dg and du; x: da.
template <typename T, int KEEP>
__device__ __forceinline__ void finish_back(const TileArgs& a, const TileProblem& p, int64_t row,
                                            const Piece8& at, bool in, float (&x)[8],
                                            const Kept8<T, KEEP>& kept_g,
                                            const Kept8<T, KEEP>& kept_u) {
  if (!in || at.col >= p.pad_i) return;
  float g[8], u[8], v[8];
  kept_g.values(g);
  kept_u.values(u);
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    float act, slope;
    gate_fn(a.gate, Kind<T>::kParts == 1, g[r], act, slope);
    v[r] = act * u[r];
    g[r] = x[r] * act;
    x[r] *= u[r] * slope;
  }
  if (p.out) put_operand<T>(p, p.out, row, at, v);
  if (a.dg) put_operand<T>(p, a.dg, row, at, x);
  if (a.du) put_operand<T>(p, a.du, row, at, g);
}

// The sums of a block that shares its tile's k.  which: 0, or 1 for u of EPI_GATE.
template <int ARRAYS>
__device__ __forceinline__ void put_part(const TileProblem& p, int split, int which, int64_t row,
                                         const Piece8& at, const float (&x)[8]) {
  float* to = p.part + ((int64_t)(split * ARRAYS + which) * p.J + row) * p.part_ld;
  store_row<float, 8>(to + (at.token * (uint32_t)p.part_ld + at.col), p.I - at.col, x);
}

// LDS of a tile: units of one operand each.
template <bool AKS, bool BKS, int BI, int BJ, int AHEAD>
struct Units {
  static constexpr int kA = Lay<AKS, BI>::kBytes, kB = Lay<BKS, BJ>::kBytes;
  static constexpr int kUnit = kA > kB ? kA : kB;
  static constexpr int kCount = 2 * AHEAD + 3;
};

// The tile of block b of a product's n: tiles come in an order that gives each of the 8 XCDs (blocks
// are dealt to them in turn) a run of neighbouring ones, which share operands in its L2.
__device__ __forceinline__ int tile_of_block(int b, int n) {
  const int x = b & 7, per = n >> 3, more = n & 7;
  return x * per + min(x, more) + (b >> 3);
}

// One tile of BI x BJ outputs, WI x WJ waves.  EPI_GATE: the tile's A rows are BI / 2 of Wg and the
// same BI / 2 of Wu, and a wave owns both projections of its features.
// KEEP: what was kept (EPI_BACK), 0 or 8.  AHEAD: whole tiles on their way.  id: of the problem's
// tiles, times its splits.
template <typename T, bool AKS, bool BKS, int EPI, int KEEP, int BI, int BJ, int WI, int WJ,
          int AHEAD>
__device__ __forceinline__ void ffn_tile(const TileArgs& a, const TileProblem& p, int id,
                                         char* lds) {
  constexpr int kThreads = WI * WJ * 64;
  constexpr int FI = BI / WI / 16, FJ = BJ / WJ / 16;  // fragments of a wave
  using U = Units<AKS, BKS, BI, BJ, AHEAD>;
  constexpr int kTileA = U::kA, kUnit = U::kUnit, kUnits = U::kCount;
  constexpr int kFeat = EPI == EPI_GATE ? BI / 2 : BI;  // features a tile

  // the larger tile's other epilogues leave no registers for sums that are put down
  constexpr bool kMaySplit = EPI == EPI_STORE || BI < 256;
  int split = 0;
  if constexpr (kMaySplit) {
    split = id / (p.tiles_i * p.tiles_j);
    id -= split * (p.tiles_i * p.tiles_j);
  }
  // columns of 8 token tiles; 4 and 16 within 1 %, 32 up to a quarter slower
  constexpr int kBand = 8;
  const int band = id / (kBand * p.tiles_i), in_band = id - band * kBand * p.tiles_i;
  const int height = min(kBand, p.tiles_j - band * kBand);
  const int ti = in_band / height, tj = band * kBand + in_band - ti * height;
  const int i0 = ti * kFeat, j0 = tj * BJ;

  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wi = wave / WJ, wj = wave % WJ;

  constexpr int RA = EPI == EPI_GATE ? BI / 2 : BI;
  Bringer<AKS, RA, kThreads> bring_a;
  Bringer<BKS, BJ, kThreads> bring_b;
  bring_a.init(p.lda, p.I - i0);
  bring_b.init(p.ldb, p.J - j0);
  Reader<AKS, BI> read_a;
  Reader<BKS, BJ> read_b;
  read_a.init(EPI == EPI_GATE ? wi * (BI / 2 / WI) : wi * (BI / WI));
  read_b.init(wj * (BJ / WJ));

  f32x4 acc[FI][FJ];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < FJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int K = max(p.KA, p.KB);
  const int per_seg = (K + kBK - 1) / kBK;
  int steps = per_seg * p.nseg, first_seg = 0, first_k = 0;
  if constexpr (kMaySplit) {
    if (p.splits > 1) {
      const int each = (steps + p.splits - 1) / p.splits, from = min(split * each, steps);
      steps = min(each, steps - from);
      if (steps > 0) first_seg = from / per_seg, first_k = from % per_seg;
    }
  }
  const int64_t corner_a = AKS ? (int64_t)i0 * 2 : (int64_t)i0 * p.lda;
  const int64_t corner_b = BKS ? (int64_t)j0 * 2 : (int64_t)j0 * p.ldb;
  const int64_t next_a = AKS ? kBK * p.lda : kBK * 2, next_b = BKS ? kBK * p.ldb : kBK * 2;

  // The operands' tiles A0 B0 A1 B1 ... take the units in turn; each has its next place in memory.
  struct Next {
    int seg, left;  // k that exist from the tile on; none are left after the last segment
    const char *p, *p2;
    uint32_t to;
  };
  const uint32_t first = base + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 1024;
  const uint32_t end = first + kUnits * kUnit;
  Next na{first_seg, p.KA - first_k * kBK, p.A[first_seg] + corner_a + first_k * next_a, nullptr,
          first};
  Next nb{first_seg, p.KB - first_k * kBK, p.B[first_seg] + corner_b + first_k * next_b,
          nullptr, first + kUnit};
  if constexpr (EPI == EPI_GATE) na.p2 = a.A2[first_seg] + corner_a + first_k * next_a;
  constexpr int kCopiesA = (EPI == EPI_GATE ? 2 : 1) * decltype(bring_a)::kLoads;
  constexpr int kCopiesB = decltype(bring_b)::kLoads;
  auto bring_a_part = [&](int r) {
    constexpr int kHalf = decltype(bring_a)::kLoads;
    if (EPI == EPI_GATE && r >= kHalf)
      bring_a.bring(na.p2, na.left, na.to + kTileA / 2, r - kHalf);
    else
      bring_a.bring(na.p, na.left, na.to, r);
  };
  auto bring_b_part = [&](int r) { bring_b.bring(nb.p, nb.left, nb.to, r); };
  auto unit_on = [&](uint32_t& u) {
    u += 2 * kUnit;
    if (u >= end) u -= kUnits * kUnit;
  };
  auto next_a_tile = [&]() {
    unit_on(na.to);
    na.p += next_a;
    if constexpr (EPI == EPI_GATE) na.p2 += next_a;
    na.left -= kBK;
    if (na.left <= 0 && na.seg + 1 < p.nseg) {
      ++na.seg;
      na.left = p.KA;
      na.p = p.A[na.seg] + corner_a;
      if constexpr (EPI == EPI_GATE) na.p2 = a.A2[na.seg] + corner_a;
    }
  };
  auto next_b_tile = [&]() {
    unit_on(nb.to);
    nb.p += next_b;
    nb.left -= kBK;
    if (nb.left <= 0 && nb.seg + 1 < p.nseg) {
      ++nb.seg;
      nb.left = p.KB;
      nb.p = p.B[nb.seg] + corner_b;
    }
  };
  struct Frags {
    s16x8 a[FI], b[FJ];
  };
  uint32_t from_a = base, from_b = base + kUnit;  // of the tile that is read
  auto unit_read = [&](uint32_t& u) {
    u += 2 * kUnit;
    if (u >= base + kUnits * kUnit) u -= kUnits * kUnit;
  };
  // 32 k: multiplies `now`, reads `next` and issues copies, all three spread over the rows of
  // fragments: a copy that finds the address unit busy holds back what its wave issues next.
  auto half = [&](const Frags& now, Frags& next, int ks, auto copies, auto&& copy) {
    constexpr int kCopies = decltype(copies)::value;
#pragma unroll
    for (int i = 0; i < FI; ++i) {
      if (i < FJ) next.b[i] = read_b.read(from_b, i, ks);
      if constexpr (EPI == EPI_GATE)
        next.a[i] = read_a.read(from_a + (i >= FI / 2 ? kTileA / 2 : 0), i % (FI / 2), ks);
      else
        next.a[i] = read_a.read(from_a, i, ks);
#pragma unroll
      for (int r = i * kCopies / FI; r < (i + 1) * kCopies / FI; ++r) copy(r);
#pragma unroll
      for (int j = 0; j < FJ; ++j) Mfma<typename Kind<T>::Half>::add(now.a[i], now.b[j], acc[i][j]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // A lane holds four consecutive features (4 (lane / 16) + 0..3 of 16) of token lane % 16.  The
  // wave turns kDump times 16 tokens at a time in LDS of its own, so that a lane gets 8
  // consecutive features and neighbouring lanes the features beside them.
  constexpr int kWide = BI / WI;                  // accumulated rows of the wave
  constexpr int kPieces = kFeat / WI / 8;         // pieces of 8 features a token
  constexpr int kRow = kWide + 4;                 // floats; 4 more keep the banks apart
  constexpr int kFit = kUnits * kUnit / (WI * WJ * 16 * kRow * 4);
  constexpr int kDump = kFit >= FJ ? FJ : kFit >= FJ / 2 ? FJ / 2 : 1;
  static_assert(kFit >= 1 && FJ % kDump == 0, "the turned tokens fit the units");
  float* turn = (float*)lds + wave * kDump * 16 * kRow;
  const int lane = threadIdx.x & 63, q = lane >> 4;
  const int iw = i0 + wi * (kFeat / WI), jw = j0 + wj * (BJ / WJ);
  constexpr int kTimes = kPieces * 16 / 64;  // pieces a lane of 16 tokens
  const int f = (lane % kPieces) * 8;
  Piece8 at;
  at.col = iw + f;
  at.token = lane / kPieces;
  at.q = at.token * groups_of(p.I) * kGroup + at.col;
  at.e = at.token * groups_of(p.I) + at.col / kGroup;
  constexpr int kTokens = 64 / kPieces;  // the tokens of the wave's next pieces lie so far on
  Kept8<T, KEEP> kg[kTimes], ku[kTimes];
  auto load_kept = [&](int j) {
#pragma unroll
    for (int c = 0; c < kTimes; ++c) {
      kg[c].load(p, a.g, a.ge, jw + j * 16 + c * kTokens, at);
      ku[c].load(p, a.u, a.ue, jw + j * 16 + c * kTokens, at);
    }
  };

  // Step n: tile n is there; after its B, which was issued in step n - AHEAD, came AHEAD more of A
  // and AHEAD - 1 of B, which may still be on their way.  Every wave has read tile n - 1, whose
  // units take B of n + AHEAD and A of n + AHEAD + 1.  The second half of tile n - 1 is multiplied
  // while the first of tile n is read.
  {
    Frags f0, f1;
#pragma unroll
    for (int i = 0; i < FI; ++i) f1.a[i] = s16x8{};
#pragma unroll
    for (int j = 0; j < FJ; ++j) f1.b[j] = s16x8{};
#pragma unroll
    for (int ahead = 0; ahead <= AHEAD; ++ahead) {
#pragma unroll
      for (int r = 0; r < kCopiesA; ++r) bring_a_part(r);
      next_a_tile();
      if (ahead == AHEAD) break;
#pragma unroll
      for (int r = 0; r < kCopiesB; ++r) bring_b_part(r);
      next_b_tile();
    }
#pragma unroll 1
    for (int n = 0; n < steps; ++n) {
      wait_copies<(AHEAD - 1) * (kCopiesA + kCopiesB) + kCopiesA>();
      half(f1, f0, 0, std::integral_constant<int, kCopiesB>{}, bring_b_part);
      next_b_tile();
      half(f0, f1, 1, std::integral_constant<int, kCopiesA>{}, bring_a_part);
      next_a_tile();
      unit_read(from_a);
      unit_read(from_b);
    }
    if constexpr (EPI == EPI_BACK) load_kept(0);
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
      for (int j = 0; j < FJ; ++j) Mfma<typename Kind<T>::Half>::add(f1.a[i], f1.b[j], acc[i][j]);
  }
  wait_all();  // nobody reads the last tile any more
#pragma unroll
  for (int j0 = 0; j0 < FJ; j0 += kDump) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the tokens before these are read
#pragma unroll
    for (int d = 0; d < kDump; ++d)
#pragma unroll
      for (int i = 0; i < FI; ++i)
        *(f32x4*)(turn + (d * 16 + (lane & 15)) * kRow + i * 16 + q * 4) = acc[i][j0 + d];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the other lanes' values are there
#pragma unroll 1
    for (int j = j0; j < j0 + kDump; ++j) {
      const float* turned = turn + j % kDump * 16 * kRow;
      Kept8<T, KEEP> g0[kTimes], u0[kTimes];
      if constexpr (EPI == EPI_BACK) {  // the next tokens' are on their way meanwhile
#pragma unroll
        for (int c = 0; c < kTimes; ++c) g0[c] = kg[c], u0[c] = ku[c];
        if (j + 1 < FJ) load_kept(j + 1);
      }
      auto piece = [&](int c, const Kept8<T, KEEP>& kept_g, const Kept8<T, KEEP>& kept_u) {
        const int t = at.token + c * kTokens;
        const int64_t row = jw + j * 16 + c * kTokens;
        const bool in = row + at.token < p.J;
        float x[8];
        read8(turned + t * kRow + f, x);
        if constexpr (EPI == EPI_STORE) {
          if (!in) return;
          if (p.splits > 1)
            put_part<1>(p, split, 0, row, at, x);
          else
            put_output<T>(p, p.out, p.ldo, row, at, x);
        } else if constexpr (EPI == EPI_GATE) {
          float u[8];
          read8(turned + t * kRow + kPieces * 8 + f, u);
          if (kMaySplit && p.splits > 1) {
            if (!in) return;
            put_part<2>(p, split, 0, row, at, x);
            put_part<2>(p, split, 1, row, at, u);
          } else {
            finish_gate<T>(a, p, row, at, in, x, u);
          }
        } else {
          if (kMaySplit && p.splits > 1) {
            if (in) put_part<1>(p, split, 0, row, at, x);
          } else {
            finish_back<T, KEEP>(a, p, row, at, in, x, kept_g, kept_u);
          }
        }
      };
      if constexpr (Kind<T>::kParts == 1) {
#pragma unroll
        for (int c = 0; c < kTimes; ++c) {
          piece(c, g0[c], u0[c]);
          __builtin_amdgcn_sched_barrier(0);  // two at once need more registers than there are
        }
      } else {  // three parts an output: too much code to be unrolled
#pragma unroll 1
        for (int c = 0; c < kTimes; ++c) {
          Kept8<T, KEEP> kept_g, kept_u;
#pragma unroll
          for (int cc = 0; cc < kTimes; ++cc)
            if (cc == c) kept_g = g0[cc], kept_u = u0[cc];
          piece(c, kept_g, kept_u);
        }
      }
    }
  }
}

// One product with its epilogue.
//
// Bound by the matrix instructions (busy 61 to 70 % of the cycles at 8192 tokens, 4096 x 10944 in
// bf16: gate and up 1.22 ms, 1200 TFLOP/s; down 0.54 ms, 1360; loops of 30 calls), and, for da, by
// its epilogue (0.80 ms, 920 TFLOP/s, busy 46 %): there all CUs come to read what was kept and to
// write three operands at the same time, 0.72 GB in all.  Few tokens are bound by the weights' bytes
// (24 tokens of 2048 x 5504: 3.1 TB/s in gate and up, 4.1 in down).
template <typename T, bool AKS, bool BKS, int EPI, int KEEP, int SIZE, int WI, int WJ, int AHEAD>
__global__ __launch_bounds__(WI* WJ * 64, 2) void k_ffn_tile(TileArgs a) {
  using U = Units<AKS, BKS, SIZE, SIZE, AHEAD>;
  __shared__ __align__(256) char lds[U::kCount * U::kUnit];
  ffn_tile<T, AKS, BKS, EPI, KEEP, SIZE, SIZE, WI, WJ, AHEAD>(
      a, a.prob[0], tile_of_block(blockIdx.x, gridDim.x), lds);
}

// The gradients, which do not depend on one another: dx (long sums) before dWg, dWu and dWd, so
// that the shorter ones fill what it leaves.  Bound by the matrix instructions at 8192 tokens (4096
// x 10944 in bf16: 2.84 ms, 1290 TFLOP/s); 777 x 1001 x 2731 in f16 34 us, 45 in three launches.
template <typename T, int SIZE, int WI, int WJ>
__global__ __launch_bounds__(WI* WJ * 64, 2) void k_ffn_grads(TileArgs a) {
  using U = Units<true, true, SIZE, SIZE, 1>;
  __shared__ __align__(256) char lds[U::kCount * U::kUnit];
  int which = 0;
  while (which + 1 < a.count && blockIdx.x >= a.prob[which + 1].first) ++which;
  const TileProblem& p = a.prob[which];
  const int id =
      tile_of_block(blockIdx.x - p.first, p.tiles_i * p.tiles_j * p.splits);
  if (p.b_strided)
    ffn_tile<T, true, true, EPI_STORE, 0, SIZE, SIZE, WI, WJ, 1>(a, p, id, lds);
  else
    ffn_tile<T, true, false, EPI_STORE, 0, SIZE, SIZE, WI, WJ, 1>(a, p, id, lds);
}

// Adds the sums of the blocks that shared a tile's k, in order, for all split products of a call.
// Bound by bytes (100 MB of sums and 40 MB out: 38 us).
struct JoinJob {
  const float* part;
  void* out;
  int64_t part_ld, ldo, J;
  int I, splits;
  unsigned first;  // block
};
struct JoinJobs {
  JoinJob job[kMaxProblems];
  int count;
};

template <typename W>
__global__ __launch_bounds__(256) void k_ffn_join(JoinJobs jobs) {
  int j = 0;
  while (j + 1 < jobs.count && blockIdx.x >= jobs.job[j + 1].first) ++j;
  const JoinJob& o = jobs.job[j];
  const int per_row = (o.I + 7) / 8;
  const int64_t first = (int64_t)(blockIdx.x - o.first) * 256, row0 = first / per_row;
  const uint32_t at = (uint32_t)(first - row0 * per_row) + threadIdx.x;
  const uint32_t down = at / (uint32_t)per_row;
  const int64_t row = row0 + down;
  const int col = (int)(at - down * (uint32_t)per_row) * 8;
  if (row >= o.J) return;
  float sum[8] = {};
  const float* from = o.part + row * o.part_ld + col;
  const int64_t next = o.J * o.part_ld;
  for (int s = 0; s < o.splits; s += 4) {  // four on their way; past the end the last one again
    float x[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      load_row<float, 8>(from + min(s + i, o.splits - 1) * next, 8, x[i]);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (s + i < o.splits) {
#pragma unroll
        for (int r = 0; r < 8; ++r) sum[r] += x[i][r];
      }
  }
  store_row<W, 8>((W*)o.out + row * o.ldo + col, o.I - col, sum);
}

// The epilogue of a gate product whose tiles' k was shared.  Bound by bytes.
template <typename T, int EPI, int KEEP>
__global__ __launch_bounds__(256) void k_ffn_finish(TileArgs a) {
  const TileProblem& p = a.prob[0];
  constexpr int kArrays = EPI == EPI_GATE ? 2 : 1;
  const int groups = groups_of(p.I), per_row = groups * 4;  // groups of lanes stay together
  const int64_t first = (int64_t)blockIdx.x * 256, row0 = first / per_row;
  const uint32_t from = (uint32_t)(first - row0 * per_row) + threadIdx.x;
  Piece8 at;
  at.token = from / (uint32_t)per_row;
  at.col = (int)(from - at.token * (uint32_t)per_row) * 8;
  at.q = at.token * groups * kGroup + at.col;
  at.e = at.token * groups + at.col / kGroup;
  const bool in = row0 + at.token < p.J;
  Kept8<T, KEEP> kg, ku;
  if constexpr (EPI == EPI_BACK) {
    kg.load(p, a.g, a.ge, row0, at);
    ku.load(p, a.u, a.ue, row0, at);
  }
  float sum[kArrays][8] = {};
  if (in && at.col < p.I) {
    const float* part = p.part + (row0 + at.token) * p.part_ld + at.col;
    const int64_t next = p.J * p.part_ld;
    for (int s = 0; s < p.splits; s += 4) {  // four on their way; past the end the last one again
      float x[4][kArrays][8];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int w = 0; w < kArrays; ++w)
          load_row<float, 8>(part + ((int64_t)min(s + i, p.splits - 1) * kArrays + w) * next,
                             p.I - at.col, x[i][w]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (s + i < p.splits) {
#pragma unroll
          for (int w = 0; w < kArrays; ++w)
#pragma unroll
            for (int r = 0; r < 8; ++r) sum[w][r] += x[i][w][r];
        }
    }
  }
  if constexpr (EPI == EPI_GATE)
    finish_gate<T>(a, p, row0, at, in, sum[0], sum[1]);
  else
    finish_back<T, KEEP>(a, p, row0, at, in, sum[0], kg, ku);
}

// Copies [rows][n] into [rows][ld] 16-bit operands, columns from n to ld cleared; a 32-bit source
// becomes three bf16 parts, a packed one (8 bits) is read back.  All operands of a call in one
// launch: they are often small, and a launch then costs more than the copy.  Bound by bytes (39 MB
// of floats into 58 MB of parts: 23 us, 4.3 TB/s).
struct OperandJob {
  const void* x;
  const uint8_t* exps;  // of a packed source (x: its int8 values), which one part holds
  int64_t ldx, rows, plane;
  void* out;
  int n, ld;
  unsigned first;  // block
};
constexpr int kMaxJobs = 5;
struct OperandJobs {
  OperandJob job[kMaxJobs];
  int count;
};

template <typename T>
__global__ __launch_bounds__(256) void k_ffn_operands(OperandJobs jobs) {
  using H = typename Kind<T>::Half;
  using W = typename Kind<T>::Whole;
  int j = 0;
  while (j + 1 < jobs.count && blockIdx.x >= jobs.job[j + 1].first) ++j;
  const OperandJob& o = jobs.job[j];
  const int per_row = o.ld / 8;
  const int64_t first = (int64_t)(blockIdx.x - o.first) * 256, row0 = first / per_row;
  const uint32_t at = (uint32_t)(first - row0 * per_row) + threadIdx.x;
  const uint32_t down = at / (uint32_t)per_row;
  const int64_t row = row0 + down;
  const int col = (int)(at - down * (uint32_t)per_row) * 8;
  if (row >= o.rows) return;
  float v[8], p[8];  // p: a part
  if (o.exps) {
    const int groups = groups_of(o.n);
    unpack8_as<H>(load_global<u32x2>((const int8_t*)o.x + row * groups * kGroup + col),
                  load_global<uint8_t>(o.exps + row * groups + col / kGroup), v);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (col + i >= o.n) v[i] = 0.f;
    store_row<H, 8>((H*)o.out + row * o.ld + col, 8, v);
    return;
  }
  load_row_end<W, 8>((const W*)o.x + row * o.ldx + col, o.n - col, v);
  if constexpr (Kind<T>::kParts == 1) {
    store_row<H, 8>((H*)o.out + row * o.ld + col, 8, v);
  } else {
#pragma unroll
    for (int part = 0; part < Kind<T>::kParts; ++part) {
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = take_part(v[i], part == 0);
      store_row<H, 8>((H*)o.out + part * o.plane + row * o.ld + col, 8, p);
    }
  }
}

}  // namespace lm
