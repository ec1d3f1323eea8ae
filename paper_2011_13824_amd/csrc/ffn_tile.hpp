// Matrix products of the gated feed-forward block on 16-bit matrix instructions.
//
//   C[j][i] = sum over segments s and k of A_s(i, k) * B_s(j, k),  32-bit sums
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
//   dWg, dWu      A = x (k-strided)              B = dg, du (k-strided)    EPI_STORE, two batches
//   dWd           A = act(g) u (k-strided)       B = dout (k-strided)      EPI_STORE
//
// 32-bit operands are three bf16 parts (hi + mid + lo = 24 bits); a product is then six segments,
// those of the largest parts, smallest first, and the error stays that of a 32-bit sum.
#pragma once

#include "lm_types.hpp"

namespace lm {

enum Epi { EPI_STORE, EPI_GATE, EPI_BACK };
enum Gate { RELU = 0, SILU = 1, GELU = 2 };

constexpr int kMaxSegs = 12;
constexpr int kBK = 64;  // k a tile step: 128 bytes of a k-contiguous row

struct TileArgs {
  const char* A[kMaxSegs];
  const char* A2[kMaxSegs];     // EPI_GATE: the rows of Wu
  const char* B[2][kMaxSegs];   // per batch
  int64_t lda, ldb;             // bytes between rows
  int64_t lda2;
  int nseg;
  int KA, KB;                   // k extents (equal up to the zero padding of a packed operand)
  int I, J;                     // output sizes
  int tiles_i, tiles_j, batches;
  // output: 16-bit or float; parts = 3 writes bf16 parts at distance `plane` elements
  void* out[2];
  int64_t ldo;                  // elements
  int pad_i;                    // columns [I, pad_i) of 16-bit operand outputs are written as 0
  int parts;
  int64_t plane;
  // gate epilogues
  int gate, keep;               // keep: -1, 0, 8
  void *g, *u;                  // what is kept: [J][I] or packed
  uint8_t *ge, *ue;             // exponents of the packed form
  void *dg, *du;                // EPI_BACK
};

__device__ __forceinline__ int up32(int n) { return (n + 31) & ~31; }

__device__ __forceinline__ void read8(const float* p, float (&x)[8]) {
  const f32x4 lo = *(const f32x4*)p, hi = *(const f32x4*)(p + 4);
#pragma unroll
  for (int r = 0; r < 4; ++r) x[r] = lo[r], x[4 + r] = hi[r];
}

template <typename T>
struct Mfma;
template <>
struct Mfma<bf16> {
  typedef bf16 x8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 mac(x8 a, x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mfma<f16> {
  typedef f16 x8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 mac(x8 a, x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};

// act(x) and act'(x).
__device__ __forceinline__ void gate_fn(int gate, float x, float& act, float& slope) {
  if (gate == RELU) {
    act = fmaxf(x, 0.f);
    slope = x > 0.f ? 1.f : 0.f;
    if (x != x) act = slope = x;
  } else if (gate == SILU) {
    const float p = 1.f / (1.f + expf(-x));
    act = x * p;
    slope = p * (1.f + x * (1.f - p));
  } else {
    const float p = 0.5f * erfcf(-0.70710678118654752f * x);
    act = x * p;
    slope = p + x * (0.39894228040143268f * expf(-0.5f * x * x));
  }
}

// 16 bytes from global memory straight into LDS, lane l's at `lds` + 16 l (`lds` is uniform).  An
// offset of kOutside is past the descriptor's end, and brings zeros.  The compiler does not see
// these as loads: wait_all() stands between them and the reads.
constexpr uint32_t kOutside = 0x80000000u;
constexpr uint32_t kExtent = 0x7fffffffu;

__device__ __forceinline__ u32x4 descriptor(const char* p) {
  const uint64_t a = (uint64_t)p;
  u32x4 d;
  d[0] = (uint32_t)a;
  d[1] = (uint32_t)(a >> 32) & 0xffffu;
  d[2] = kExtent;
  d[3] = 0x00020000u;
  return d;
}
__device__ __forceinline__ void bring16(u32x4 desc, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds),
               "v"(offset), "s"(desc)
               : "memory");
}
__device__ __forceinline__ void wait_all() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) s16x8 lds_s16x8;

// Where an operand's tile (R rows of i or j, kBK of k) lies in LDS.
//   k-contiguous: row r is 8 pieces of 16 bytes, piece p at p ^ (r / 2 % 8): the 16 rows that one
//   read takes then start in 16 different 16-byte columns of the 256 bytes of banks.
//   k-strided: line k is R / 8 pieces, piece p at p ^ 2 f(k), f(k) = k % 4 + 4 (k / 8 % 2): a
//   transposing read takes 32 bytes of 4 lines, from 2 groups of lanes at k and k + 8.
template <bool KS, int R>
struct Lay {
  static constexpr int kPieces = KS ? R / 8 : kBK / 8;  // of a line
  static constexpr int kBytes = R * kBK * 2;
  static __device__ __forceinline__ int swizzle(int line) {
    return KS ? ((line & 3) | ((line >> 3) & 1) << 2) << 1 : (line >> 1) & 7;
  }
};

// One operand's copies: thread t of THREADS brings pieces t, t + THREADS, ... of a tile.
template <bool KS, int R, int THREADS>
struct Bringer {
  using L = Lay<KS, R>;
  static constexpr int kLoads = L::kBytes / 16 / THREADS;
  uint32_t off[kLoads];  // byte offsets from the tile's corner; kOutside for rows past the end
  int kk[kLoads];        // first k of the piece (k-contiguous) or the line's k

  // `rows`: valid rows from the tile's corner on.
  __device__ __forceinline__ void init(int64_t ld, int rows) {
#pragma unroll
    for (int r = 0; r < kLoads; ++r) {
      const int c = r * THREADS + threadIdx.x;
      const int line = c / L::kPieces, p = (c % L::kPieces) ^ L::swizzle(line);
      const bool in = KS ? p * 8 < rows : line < rows;
      off[r] = in ? (uint32_t)(line * ld) + p * 16 : kOutside;
      kk[r] = KS ? line : p * 8;
    }
  }
  // Brings k from the tile's step on, `left` of which exist.
  __device__ __forceinline__ void bring(const char* base, int left, uint32_t lds,
                                        int r0 = 0, int r1 = kLoads) const {
    const u32x4 d = descriptor(base);
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 1024;
#pragma unroll
    for (int r = 0; r < kLoads; ++r) {
      if (r < r0 || r >= r1) continue;
      const uint32_t o = left >= kBK || kk[r] < left ? off[r] : kOutside;
      bring16(d, o, lds + r * THREADS * 16 + wave);
    }
  }
};

// A fragment: 8 k of one row per lane (row = lane % 16, k = 8 (lane / 16) + 0..7 of 32).
template <bool KS, int R>
struct Reader {
  using L = Lay<KS, R>;
  uint32_t at[KS ? R / 16 : 2];
  // `row0`: the wave's first row in the tile; fragments lie 16 rows apart.
  __device__ __forceinline__ void init(int row0, int frags) {
    const int lane = threadIdx.x & 63, m = lane & 15, q = lane >> 4;
    if constexpr (KS) {
      const int k = q * 8 + (m >> 2);
#pragma unroll
      for (int f = 0; f < R / 16; ++f)
        if (f < frags) {
          const int p = (row0 + f * 16) / 8 + ((m & 3) >> 1);
          at[f] = k * R * 2 + (p ^ L::swizzle(k)) * 16 + (m & 1) * 8;
        }
    } else {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
        at[ks] = (row0 + m) * 128 + ((ks * 4 + q) ^ L::swizzle(m)) * 16;
    }
  }
  __device__ __forceinline__ s16x8 read(uint32_t tile, int f, int ks) const {
    if constexpr (KS) {
      const uint32_t a = tile + at[f] + ks * 32 * R * 2;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)a);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(a + 4 * R * 2));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      return *(lds_s16x8*)(uintptr_t)(tile + at[ks] + f * 2048);
    }
  }
};

// Eight consecutive features of a token, at any alignment of the output's rows.

// An operand of a later product: 16 bits, or three bf16 parts of a 32-bit value.  The columns
// [I, pad_i) are cleared.
template <typename T>
__device__ __forceinline__ void put_operand(const TileArgs& a, void* base, int64_t row, int col,
                                            const float (&v)[8]) {
  T* p = (T*)base + row * a.ldo + col;
  float x[8], rest[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) rest[r] = col + r < a.I ? v[r] : 0.f;
  if (a.parts == 1) {
    store_row<T, 8>(p, a.pad_i - col, rest);
    return;
  }
#pragma unroll
  for (int part = 0; part < 3; ++part) {
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      x[r] = (float)(T)rest[r];
      rest[r] -= x[r];
      if (!(fabsf(rest[r]) < INFINITY)) rest[r] = 0.f;  // the remainder of an infinity or a NaN
    }
    store_row<T, 8>(p + part * a.plane, a.pad_i - col, x);
  }
}

template <typename T>
__device__ __forceinline__ void put_output(const TileArgs& a, void* base, int64_t ld, int64_t row,
                                           int col, const float (&v)[8]) {
  if (a.parts == 3)
    store_row<float, 8>((float*)base + row * ld + col, a.I - col, v);
  else
    store_row<T, 8>((T*)base + row * ld + col, a.I - col, v);
}

// What the forward pass keeps: packed with a scale for 32 features (four neighbouring lanes), or
// as it is.  Every lane of the wave comes here.
template <typename T>
__device__ __forceinline__ void keep8(const TileArgs& a, void* base, uint8_t* exps, int64_t row,
                                      int col, const float (&v)[8]) {
  const bool in = row < a.J && col < up32(a.I);
  if (a.keep != 8) {
    if (in) put_output<T>(a, base, a.I, row, col, v);
    return;
  }
  uint32_t top = 0;
#pragma unroll
  for (int r = 0; r < 8; ++r)
    if (col + r < a.I) top = max(top, magnitude(v[r]));
  top = max(top, (uint32_t)__shfl_xor((int)top, 1));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2));
  const int e = group_exponent(top);
  const float inv = group_inverse(e);
  const int groups = groups_of(a.I);
  if (!in) return;
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int r = 0; r < 8; ++r)
    if (col + r < a.I) w[r >> 2] |= (uint32_t)(to_int8(v[r], inv) & 255) << 8 * (r & 3);
  *(uint2*)((int8_t*)base + row * groups * kGroup + col) = make_uint2(w[0], w[1]);
  if ((col & 31) == 0) exps[row * groups + col / kGroup] = (uint8_t)e;
}

template <typename T>
__device__ __forceinline__ void kept8(const TileArgs& a, const void* base, const uint8_t* exps,
                                      int64_t row, int col, float (&v)[8]) {
  if (a.keep == 8) {
    const int groups = groups_of(a.I);
    const uint2 w = *(const uint2*)((const int8_t*)base + row * groups * kGroup + col);
    const float s = group_scale(exps[row * groups + col / kGroup]);
#pragma unroll
    for (int r = 0; r < 8; ++r) v[r] = (float)(int8_t)((r < 4 ? w.x : w.y) >> 8 * (r & 3)) * s;
  } else if (a.parts == 3) {
    load_row<float, 8>((const float*)base + row * a.I + col, a.I - col, v);
  } else {
    load_row<T, 8>((const T*)base + row * a.I + col, a.I - col, v);
  }
}

// BI x BJ output tile, WI x WJ waves.  EPI_GATE: the tile's A rows are BI / 2 of Wg and the same
// BI / 2 of Wu, and a wave owns both projections of its features.
template <typename T, bool AKS, bool BKS, int EPI, int BI, int BJ, int WI, int WJ>
__global__ __launch_bounds__(WI* WJ * 64, WI* WJ == 8 ? 2 : 2) void k_ffn_tile(TileArgs a) {
  constexpr int kThreads = WI * WJ * 64;
  constexpr int FI = BI / WI / 16, FJ = BJ / WJ / 16;  // fragments of a wave
  constexpr int kTileA = Lay<AKS, BI>::kBytes, kTileB = Lay<BKS, BJ>::kBytes;
  constexpr int kStage = kTileA + kTileB;
  constexpr int kFeat = EPI == EPI_GATE ? BI / 2 : BI;  // features a tile
  __shared__ __align__(256) char lds[2 * kStage];

  // tiles in an order that gives each of the 8 XCDs (blocks are dealt to them in turn) a run of
  // neighbouring tiles, in columns of 8 token tiles: they share operands in its L2
  const int total = gridDim.x;
  int id;
  {
    const int x = blockIdx.x & 7, per = total >> 3, more = total & 7;
    id = x * per + min(x, more) + (blockIdx.x >> 3);
  }
  const int per_batch = a.tiles_i * a.tiles_j;
  const int batch = id / per_batch;
  id -= batch * per_batch;
  constexpr int kBand = 8;
  const int band = id / (kBand * a.tiles_i), in_band = id - band * kBand * a.tiles_i;
  const int height = min(kBand, a.tiles_j - band * kBand);
  const int ti = in_band / height, tj = band * kBand + in_band - ti * height;
  const int i0 = ti * kFeat, j0 = tj * BJ;

  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wi = wave / WJ, wj = wave % WJ;

  constexpr int RA = EPI == EPI_GATE ? BI / 2 : BI;
  Bringer<AKS, RA, kThreads> bring_a;
  Bringer<BKS, BJ, kThreads> bring_b;
  bring_a.init(a.lda, a.I - i0);
  bring_b.init(a.ldb, a.J - j0);
  Reader<AKS, BI> read_a;
  Reader<BKS, BJ> read_b;
  read_a.init(EPI == EPI_GATE ? wi * (BI / 2 / WI) : wi * (BI / WI), FI);
  read_b.init(wj * (BJ / WJ), FJ);

  f32x4 acc[FI][FJ];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < FJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int K = max(a.KA, a.KB);
  const int per_seg = (K + kBK - 1) / kBK, steps = per_seg * a.nseg;
  const int64_t corner_a = AKS ? (int64_t)i0 * 2 : (int64_t)i0 * a.lda;
  const int64_t corner_b = BKS ? (int64_t)j0 * 2 : (int64_t)j0 * a.ldb;
  const int64_t next_a = AKS ? kBK * a.lda : kBK * 2, next_b = BKS ? kBK * a.ldb : kBK * 2;

  int seg = 0, ks = 0;  // of the step that is brought next
  auto bring = [&](int stage) {
    const uint32_t to = base + stage * kStage;
    const int k0 = ks * kBK;
    bring_a.bring(a.A[seg] + corner_a + ks * next_a, a.KA - k0, to);
    if constexpr (EPI == EPI_GATE)
      bring_a.bring(a.A2[seg] + corner_a + ks * next_a, a.KA - k0, to + kTileA / 2);
    bring_b.bring(a.B[batch][seg] + corner_b + ks * next_b, a.KB - k0, to + kTileA);
    if (++ks == per_seg) ks = 0, ++seg;
  };

  if (steps > 0) bring(0);
  for (int step = 0; step < steps; ++step) {
    wait_all();  // this step's tile is there, and nobody reads the other stage any more
    if (step + 1 < steps) bring((step + 1) & 1);
    const uint32_t ta = base + (step & 1) * kStage, tb = ta + kTileA;
#pragma unroll
    for (int kk = 0; kk < kBK / 32; ++kk) {
      s16x8 fa[FI], fb[FJ];
#pragma unroll
      for (int j = 0; j < FJ; ++j) fb[j] = read_b.read(tb, j, kk);
#pragma unroll
      for (int i = 0; i < FI; ++i) {
        if constexpr (EPI == EPI_GATE)
          fa[i] = read_a.read(ta + (i >= FI / 2 ? kTileA / 2 : 0), i % (FI / 2), kk);
        else
          fa[i] = read_a.read(ta, i, kk);
      }
#pragma unroll
      for (int i = 0; i < FI; ++i)
#pragma unroll
        for (int j = 0; j < FJ; ++j)
          acc[i][j] = Mfma<T>::mac(__builtin_bit_cast(typename Mfma<T>::x8, fa[i]),
                                   __builtin_bit_cast(typename Mfma<T>::x8, fb[j]), acc[i][j]);
    }
  }

  // A lane holds four consecutive features (4 (lane / 16) + 0..3 of 16) of token lane % 16.  The
  // wave turns 16 tokens at a time in LDS of its own, so that a lane gets 8 consecutive features
  // and neighbouring lanes the features beside them.
  constexpr int kWide = BI / WI;                  // accumulated rows of the wave
  constexpr int kPieces = kFeat / WI / 8;         // pieces of 8 features a token
  constexpr int kRow = kWide + 4;                 // floats; 4 more keep the banks apart
  static_assert(WI * WJ * 16 * kRow * 4 <= 2 * kStage, "the turned tokens fit the stages");
  wait_all();  // nobody reads the last tile any more
  float* turn = (float*)lds + wave * 16 * kRow;
  const int lane = threadIdx.x & 63, q = lane >> 4;
  const int iw = i0 + wi * (kFeat / WI), jw = j0 + wj * (BJ / WJ);
#pragma unroll
  for (int j = 0; j < FJ; ++j) {
#pragma unroll
    for (int i = 0; i < FI; ++i)
      *(f32x4*)(turn + (lane & 15) * kRow + i * 16 + q * 4) = acc[i][j];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the other lanes' values are there
#pragma unroll 1
    for (int c = lane; c < 16 * kPieces; c += 64) {
      const int token = c / kPieces, f = (c % kPieces) * 8;
      const int64_t row = jw + j * 16 + token;
      const int col = iw + f;
      float x[8];
      read8(turn + token * kRow + f, x);
      if constexpr (EPI == EPI_STORE) {
        if (row < a.J) put_output<T>(a, a.out[batch], a.ldo, row, col, x);
      } else if constexpr (EPI == EPI_GATE) {
        float u[8];
        read8(turn + token * kRow + kPieces * 8 + f, u);
        if (a.keep >= 0) {
          keep8<T>(a, a.g, a.ge, row, col, x);
          keep8<T>(a, a.u, a.ue, row, col, u);
        }
        if (row >= a.J || col >= a.pad_i) continue;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          float act, slope;
          gate_fn(a.gate, x[r], act, slope);
          u[r] *= act;
        }
        put_operand<T>(a, a.out[0], row, col, u);
      } else {
        if (row >= a.J || col >= a.pad_i) continue;
        float g[8] = {}, u[8] = {}, v[8], du[8];
        if (col < a.I) {
          kept8<T>(a, a.g, a.ge, row, col, g);
          kept8<T>(a, a.u, a.ue, row, col, u);
        }
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          float act, slope;
          gate_fn(a.gate, g[r], act, slope);
          v[r] = act * u[r];
          du[r] = x[r] * act;
          x[r] *= u[r] * slope;
        }
        if (a.out[0]) put_operand<T>(a, a.out[0], row, col, v);
        if (a.dg) put_operand<T>(a, a.dg, row, col, x);
        if (a.du) put_operand<T>(a, a.du, row, col, du);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // read before the next tokens arrive
  }
}

// Copies [rows][n] into [rows][ld] 16-bit operands, columns from n to ld cleared; a 32-bit source
// becomes three bf16 parts.  Bound by bytes.
template <typename S, typename T, int PARTS>
__global__ __launch_bounds__(256) void k_operand(const S* __restrict__ x, int64_t ldx,
                                                 int64_t rows, int n, T* __restrict__ out, int ld,
                                                 int64_t plane) {
  const int per_row = (ld + 7) / 8;
  const int64_t first = (int64_t)blockIdx.x * 256;
  const int64_t row0 = first / per_row;
  const uint32_t at = (uint32_t)(first - row0 * per_row) + threadIdx.x;
  const uint32_t down = at / (uint32_t)per_row;
  const int64_t row = row0 + down;
  const int col = (int)(at - down * (uint32_t)per_row) * 8;
  if (row >= rows) return;
  float v[8], p[8];
  load_row<S, 8>(x + row * ldx + col, n - col, v);
#pragma unroll
  for (int part = 0; part < PARTS; ++part) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = (float)(T)v[i];
      v[i] -= p[i];
      if (!(fabsf(v[i]) < INFINITY)) v[i] = 0.f;
    }
    store_row<T, 8>(out + part * plane + row * ld + col, ld - col, p);
  }
}

}  // namespace lm
