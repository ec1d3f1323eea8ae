// Selective state space scan over sequences that lie behind each other, and its backward pass.
//
//   delta = softplus(dt + bias),  h_t = e^(delta A) h_{t-1} + delta u B_t     (per column and state)
//   v_t = sum_n C_t h_t + D u,    y = v silu(z)
//
// and with p = dy silu(z), from the last row on:
//
//   g_t = C_t p_t + e^(delta_{t+1} A) g_{t+1},  e_t = g_t e^(delta_t A) h_{t-1}
//   dC_t = sum over columns of p h_t,  dB_t = sum over columns of g_t delta u
//   du = delta sum_n g B + D p,  ddelta = sum_n e A + u sum_n g B,  ddt = ddelta sigmoid(dt + bias)
//   dA = sum_t e delta,  dD = sum_t p u,  dbias = sum_t ddt,  dz = dy v silu'(z)
//
// Bound by the vector units: every row, column and state takes an exponential (four slots) and four
// more instructions forward.  A column's states lie in LANES neighbouring lanes, four states each; a
// block takes 256 / LANES columns and walks over the rows by 16, of which it first computes what does
// not depend on the state (delta, delta u, and B and C as floats), one value a thread, into LDS.
//
// Rows are cut into chunks, so that there are enough blocks.  Before the real walk a first one
// computes what every chunk adds to a state that enters it with 0 (only for chunks whose last
// sequence goes on behind them, and from where that begins); the state that enters a chunk then
// follows from chunk to chunk, e^(A sum of delta) being what is left of the one before.  The
// gradient does the same from the last chunk on.  For it the forward pass keeps the state in front of
// every 16 rows, from which those 16 are computed again.
#pragma once

#include <type_traits>

#include "sequences.hpp"

namespace lm {

constexpr int kSpan = 16;  // rows of a step, and between the states that are kept

// What a row is, as a step's flags: it has a sequence; it is its first, its last row.
constexpr int kInside = 1, kBegins = 2, kEnds = 4;

template <typename T>
struct Scan {
  const T *u, *dt, *z, *B, *C, *dy;
  const float *A, *D, *bias, *state;
  T *y, *du, *ddt, *dz;
  float *state_out, *kept;
  int64_t ldu, lddt, ldz, ldB, ldC, ldy, lddy, lddu, ldddt, lddz;
  Sequences s;
  int n, states;        // states <= 4 * LANES
  int chunk, chunks;    // rows of a chunk, a multiple of kSpan
  // per chunk: the state that a chunk adds, then the one that enters it; that of its last sequence's
  // begin; the sum of delta.  [chunks][n][4 * LANES], [chunks][n]; one flag a chunk
  float *local, *begin, *deltas;
  int *links;           // kGoesOn, kWhole
  float *dA, *dD, *dbias;  // [chunks][n][4 * LANES], [chunks][n]: parts
  float* dBC;           // [groups][rows][2][4 * LANES]: parts
};

// A chunk's last sequence goes on in the next (or, backwards, its first one comes from the chunk
// before); it fills the whole chunk, so that the state that enters is not replaced in it.
constexpr int kGoesOn = 1, kWhole = 2;

// log(1 + e^x) and, for its slope, e^-|x|.  log(1 + v) = 2 artanh(v / (2 + v)), whose series in the
// square of that (at most 1/9) is cut where a term is under 2^-25 of the sum.
__device__ __forceinline__ float softplus(float x, float& v) {
  v = __builtin_amdgcn_exp2f(fabsf(x) * -1.44269504f);
  const float s = v * __builtin_amdgcn_rcpf(2.f + v), q = s * s;
  float r = 2.f / 15.f;
  r = fmaf(r, q, 2.f / 13.f);
  r = fmaf(r, q, 2.f / 11.f);
  r = fmaf(r, q, 2.f / 9.f);
  r = fmaf(r, q, 2.f / 7.f);
  r = fmaf(r, q, 2.f / 5.f);
  r = fmaf(r, q, 2.f / 3.f);
  r = fmaf(r, q, 2.f);
  return fmaf(s, r, fmaxf(x, 0.f));
}
__device__ __forceinline__ float softplus_slope(float x, float v) {
  return (x >= 0.f ? 1.f : v) * __builtin_amdgcn_rcpf(1.f + v);
}

// The sum over the LANES neighbouring lanes of a column; each gets it.  The second half of the steps
// mirrors, which exchanges groups that already hold one value.
template <int LANES>
__device__ __forceinline__ float column_sum(float v) {
  auto dpp = [](float x, auto ctrl) {
    return __int_as_float(
        __builtin_amdgcn_update_dpp(0, __float_as_int(x), ctrl.value, 0xf, 0xf, true));
  };
  v += dpp(v, std::integral_constant<int, 0xb1>{});  // quad_perm 1 0 3 2
  if constexpr (LANES > 2) v += dpp(v, std::integral_constant<int, 0x4e>{});   // 2 3 0 1
  if constexpr (LANES > 4) v += dpp(v, std::integral_constant<int, 0x141>{});  // row_half_mirror
  if constexpr (LANES > 8) v += dpp(v, std::integral_constant<int, 0x140>{});  // row_mirror
  return v;
}

// N values of a row of floats that may end in between.
template <int N, typename T>
__device__ __forceinline__ void load_some(const T* p, int valid, float (&v)[N]) {
  if constexpr (N == 1) {
    v[0] = valid > 0 ? (float)load_global<T>(p) : 0.f;
  } else {
    load_row_end<T, N>(p, valid, v);
  }
}
template <int N, typename T>
__device__ __forceinline__ void store_some(T* p, int valid, const float (&v)[N]) {
  if constexpr (N == 1) {
    if (valid > 0) store_global<T>(p, (T)v[0]);
  } else {
    store_row<T, N>(p, valid, v);
  }
}

// The columns and rows of a block and its threads.
template <int LANES>
struct ScanPlace {
  static constexpr int kColumns = 256 / LANES;
  static constexpr int kWide = kSpan / LANES;  // columns that a thread prepares of one row
  int first_col, col, lane;                    // of the walk
  int own_row, own_col;                        // of what the thread prepares
  __device__ __forceinline__ explicit ScanPlace(int group) {
    first_col = group * kColumns;
    col = first_col + (int)threadIdx.x / LANES;
    lane = threadIdx.x % LANES;
    own_row = (int)threadIdx.x / (kColumns / kWide);
    own_col = (int)threadIdx.x % (kColumns / kWide) * kWide;
  }
};

template <int LANES>
struct ScanShared {
  static constexpr int kColumns = 256 / LANES, kStates = 4 * LANES;
  float delta[kSpan][kColumns], du[kSpan][kColumns];
  __attribute__((aligned(16))) float B[kSpan][kStates];
  __attribute__((aligned(16))) float C[kSpan][kStates];
  float v[kSpan][kColumns];
  int flags[kSpan], slot[kSpan], plain;  // plain: 16 rows inside one sequence
};

// Flags and slots of the rows t0 .. t0 + 15, by the first 16 threads.
template <typename T, int LANES>
__device__ __forceinline__ void scan_rows(const Scan<T>& a, int64_t t0, ScanShared<LANES>& sh) {
  if (threadIdx.x >= 64) return;
  const int64_t t = t0 + threadIdx.x;
  int flags = 0;
  if (threadIdx.x < kSpan) {
    const int slot = a.s.slot(t);
    if (slot >= 0) {
      flags = kInside;
      if (t == 0 || a.s.slot(t - 1) != slot) flags |= kBegins;
      if (a.s.slot(t + 1) != slot) flags |= kEnds;
    }
    sh.flags[threadIdx.x] = flags;
    sh.slot[threadIdx.x] = slot;
  }
  const uint64_t plain = __ballot(flags == kInside);
  if (threadIdx.x == 0) sh.plain = (plain & 0xffff) == 0xffff;
}

// B and C of 16 rows as floats, 0 behind the last state and the last row.
template <typename T, int LANES>
__device__ __forceinline__ void scan_vectors(const Scan<T>& a, int64_t t0, const T* p, int64_t ld,
                                             float (&out)[kSpan][4 * LANES]) {
  for (int i = threadIdx.x; i < kSpan * 4 * LANES; i += 256) {
    const int r = i / (4 * LANES), k = i % (4 * LANES);
    float v = 0.f;
    if (t0 + r < a.s.rows && k < a.states) v = (float)load_global<T>(p + (t0 + r) * ld + k);
    out[r][k] = v;
  }
}

// Four states of a column out of [n][states] (padded: [n][4 * LANES]), 0 behind the last.
template <int LANES>
__device__ __forceinline__ void load_states(const float* p, int col, int lane, int states, int n,
                                            float (&h)[4]) {
  load_row_end<float, 4>(p + (int64_t)min(col, n - 1) * states + min(lane * 4, states - 1),
                         col < n ? states - lane * 4 : 0, h);
}
template <int LANES>
__device__ __forceinline__ void load_padded(const float* p, int64_t at, int n, int col, int lane,
                                            float (&h)[4]) {
  load_row<float, 4>(p + (at * n + min(col, n - 1)) * (4 * LANES) + lane * 4, 4, h);
}
template <int LANES>
__device__ __forceinline__ void store_padded(float* p, int64_t at, int n, int col, int lane,
                                             const float (&h)[4]) {
  if (col < n) store_row<float, 4>(p + (at * n + col) * (4 * LANES) + lane * 4, 4, h);
}

// A in powers of two a unit of delta.
template <typename T, int LANES>
__device__ __forceinline__ void load_A(const Scan<T>& a, int col, int lane, float (&A)[4]) {
  load_states<LANES>(a.A, col, lane, a.states, a.n, A);
}

// What a thread holds of a row's inputs.
template <int W>
struct ScanOwn {
  float u[W], dt[W];
};

template <typename T, int LANES>
__device__ __forceinline__ ScanOwn<ScanPlace<LANES>::kWide> scan_own(
    const Scan<T>& a, const ScanPlace<LANES>& at, int64_t t0) {
  constexpr int W = ScanPlace<LANES>::kWide;
  ScanOwn<W> o;
  const int64_t t = min(t0 + at.own_row, a.s.rows - 1);
  const int col = at.first_col + at.own_col, c = min(col, a.n - 1);
  load_some<W>(a.u + t * a.ldu + c, a.n - col, o.u);
  load_some<W>(a.dt + t * a.lddt + c, a.n - col, o.dt);
  return o;
}

template <int LANES, int W>
__device__ __forceinline__ void scan_prepare(const ScanPlace<LANES>& at, const ScanOwn<W>& o,
                                             const float (&bias)[W], ScanShared<LANES>& sh) {
#pragma unroll
  for (int i = 0; i < W; ++i) {
    float v;
    const float delta = softplus(o.dt[i] + bias[i], v);
    sh.delta[at.own_row][at.own_col + i] = delta;
    sh.du[at.own_row][at.own_col + i] = delta * o.u[i];
  }
}

// ---------------------------------------------------------------------------------------------
// Forward
// ---------------------------------------------------------------------------------------------

// What a chunk adds to the state behind it: links, local, begin, deltas.
template <typename T, int LANES>
__global__ __launch_bounds__(256) void k_scan_local(Scan<T> a, int groups) {
  constexpr int W = ScanPlace<LANES>::kWide;
  __shared__ ScanShared<LANES> sh;
  __shared__ int begins;
  const int chunk = blockIdx.x / groups, group = blockIdx.x % groups;
  const ScanPlace<LANES> at(group);
  const int64_t first = (int64_t)chunk * a.chunk, end = first + a.chunk;  // not the last chunk
  const int slot = a.s.slot(end - 1);
  const bool goes_on = slot >= 0 && a.s.slot(end) == slot;
  // the last row of the chunk in which that sequence begins, -1 if it comes from further ahead
  if (threadIdx.x == 0) begins = -1;
  __syncthreads();
  if (goes_on)
    for (int i = threadIdx.x; i < a.chunk; i += 256)
      if (first + i == 0 || a.s.slot(first + i) != a.s.slot(first + i - 1)) atomicMax(&begins, i);
  __syncthreads();
  const int from = begins;
  if (group == 0 && threadIdx.x == 0)
    a.links[chunk] = goes_on ? kGoesOn | (from < 0 ? kWhole : 0) : 0;
  if (!goes_on) return;
  float A[4], h[4] = {}, bias[W] = {};
  load_A<T, LANES>(a, at.col, at.lane, A);
#pragma unroll
  for (int i = 0; i < 4; ++i) A[i] *= 1.44269504f;
  if (a.bias)
    load_some<W>(a.bias + min(at.first_col + at.own_col, a.n - 1),
                 a.n - at.first_col - at.own_col, bias);
  if (from >= 0 && a.state) {
    load_states<LANES>(a.state + (int64_t)slot * a.n * a.states, at.col, at.lane, a.states, a.n, h);
    store_padded<LANES>(a.begin, chunk, a.n, at.col, at.lane, h);
  }
  float sum = 0.f;
  const int64_t start = first + max(from, 0);
  int64_t t0 = start / kSpan * kSpan;
  ScanOwn<W> own = scan_own<T, LANES>(a, at, t0);
  for (; t0 < end; t0 += kSpan) {
    __syncthreads();
    scan_prepare<LANES>(at, own, bias, sh);
    scan_vectors<T, LANES>(a, t0, a.B, a.ldB, sh.B);
    __syncthreads();
    own = scan_own<T, LANES>(a, at, t0 + kSpan);
    const int column = threadIdx.x / LANES;
    const int skip = (int)max((int64_t)0, start - t0);
    if (skip == 0) {
#pragma unroll
      for (int r = 0; r < kSpan; ++r) {
        const float delta = sh.delta[r][column], du = sh.du[r][column];
        sum += delta;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          h[i] = fmaf(__builtin_amdgcn_exp2f(delta * A[i]), h[i], du * sh.B[r][at.lane * 4 + i]);
      }
    } else {
      for (int r = skip; r < kSpan; ++r) {
        const float delta = sh.delta[r][column], du = sh.du[r][column];
        sum += delta;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          h[i] = fmaf(__builtin_amdgcn_exp2f(delta * A[i]), h[i], du * sh.B[r][at.lane * 4 + i]);
      }
    }
  }
  store_padded<LANES>(a.local, chunk, a.n, at.col, at.lane, h);
  if (at.lane == 0 && at.col < a.n) a.deltas[(int64_t)chunk * a.n + at.col] = sum;
}

// The states that enter the chunks, in the place of what the chunks add: that of chunk c + 1 stands
// at c.  BACK: from the last chunk on; what enters chunk c from behind stands at c + 1.
template <typename T, int LANES, bool BACK>
__global__ __launch_bounds__(256) void k_scan_link(Scan<T> a) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int col = (int)(id / LANES), lane = (int)(id % LANES);
  if (col >= a.n) return;
  float A[4], h[4] = {};
  load_A<T, LANES>(a, col, lane, A);
#pragma unroll
  for (int i = 0; i < 4; ++i) A[i] *= 1.44269504f;
  for (int i = 0; i + 1 < a.chunks; ++i) {
    const int c = BACK ? a.chunks - 1 - i : i;
    const int link = a.links[c];
    if (!(link & kGoesOn)) {
      h[0] = h[1] = h[2] = h[3] = 0.f;
      continue;
    }
    float add[4];
    load_padded<LANES>(a.local, c, a.n, col, lane, add);
    const float sum = a.deltas[(int64_t)c * a.n + col];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      h[k] = link & kWhole ? fmaf(__builtin_amdgcn_exp2f(sum * A[k]), h[k], add[k]) : add[k];
    store_padded<LANES>(a.local, c, a.n, col, lane, h);
  }
}

template <typename T, int LANES>
__global__ __launch_bounds__(256) void k_scan_fwd(Scan<T> a, int groups) {
  constexpr int W = ScanPlace<LANES>::kWide, kOwn = kSpan / LANES;
  __shared__ ScanShared<LANES> sh;
  const int chunk = blockIdx.x / groups;
  const ScanPlace<LANES> at(blockIdx.x % groups);
  const int64_t first = (int64_t)chunk * a.chunk, end = min(first + a.chunk, a.s.rows);
  const int column = threadIdx.x / LANES;
  const int own_at = at.first_col + at.own_col, own_safe = min(own_at, a.n - 1);
  const int own_valid = a.n - own_at;
  float A[4], h[4] = {}, bias[W] = {}, D[W] = {};
  load_A<T, LANES>(a, at.col, at.lane, A);
#pragma unroll
  for (int i = 0; i < 4; ++i) A[i] *= 1.44269504f;
  if (a.bias) load_some<W>(a.bias + own_safe, own_valid, bias);
  if (a.D) load_some<W>(a.D + own_safe, own_valid, D);
  if (chunk > 0 && a.links[chunk - 1] & kGoesOn)
    load_padded<LANES>(a.local, chunk - 1, a.n, at.col, at.lane, h);
  // the state of the sequence that goes on behind the chunk may have been replaced in the meantime,
  // where it goes to the place that it came from
  const bool goes_on = chunk + 1 < a.chunks && a.links[chunk] & kGoesOn;
  const int last_slot = goes_on ? a.s.slot(end - 1) : -1;
  ScanOwn<W> own = scan_own<T, LANES>(a, at, first);
  for (int64_t t0 = first; t0 < end; t0 += kSpan) {
    const int64_t mine = t0 + at.own_row;
    float z[W];
    if (a.z) load_some<W>(a.z + min(mine, a.s.rows - 1) * a.ldz + own_safe, own_valid, z);
    scan_prepare<LANES>(at, own, bias, sh);
    scan_vectors<T, LANES>(a, t0, a.B, a.ldB, sh.B);
    scan_vectors<T, LANES>(a, t0, a.C, a.ldC, sh.C);
    scan_rows<T, LANES>(a, t0, sh);
    float u[W];
#pragma unroll
    for (int i = 0; i < W; ++i) u[i] = own.u[i];
    __syncthreads();
    own = scan_own<T, LANES>(a, at, t0 + kSpan);
    const bool inside = sh.flags[at.own_row] & kInside;
    if (a.kept) store_padded<LANES>(a.kept, t0 / kSpan, a.n, at.col, at.lane, h);
    float v[kOwn];
    auto row = [&](int r) {
      const float delta = sh.delta[r][column], du = sh.du[r][column];
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        h[i] = fmaf(__builtin_amdgcn_exp2f(delta * A[i]), h[i], du * sh.B[r][at.lane * 4 + i]);
        sum = fmaf(sh.C[r][at.lane * 4 + i], h[i], sum);
      }
      return column_sum<LANES>(sum);
    };
    if (sh.plain) {
#pragma unroll
      for (int r = 0; r < kSpan; ++r) {
        const float sum = row(r);
        if (r % LANES == 0) v[r / LANES] = sum;
        v[r / LANES] = at.lane == r % LANES ? sum : v[r / LANES];
      }
    } else {
#pragma unroll
      for (int r = 0; r < kSpan; ++r) {
        const int flags = sh.flags[r], slot = sh.slot[r];
        float sum = 0.f;
        if (flags & kBegins) {
          h[0] = h[1] = h[2] = h[3] = 0.f;
          if (a.state) {
            if (slot == last_slot)
              load_padded<LANES>(a.begin, chunk, a.n, at.col, at.lane, h);
            else
              load_states<LANES>(a.state + (int64_t)slot * a.n * a.states, at.col, at.lane,
                                 a.states, a.n, h);
          }
        }
        if (flags & kInside) sum = row(r);
        if (flags & kEnds && a.state_out && at.col < a.n)
          store_row<float, 4>(a.state_out + ((int64_t)slot * a.n + at.col) * a.states + at.lane * 4,
                              a.states - at.lane * 4, h);
        if (r % LANES == 0) v[r / LANES] = sum;
        v[r / LANES] = at.lane == r % LANES ? sum : v[r / LANES];
      }
    }
#pragma unroll
    for (int i = 0; i < kOwn; ++i) sh.v[i * LANES + at.lane][column] = v[i];
    __syncthreads();
    if (mine < end) {
      float y[W];
#pragma unroll
      for (int i = 0; i < W; ++i) {
        y[i] = fmaf(D[i], u[i], sh.v[at.own_row][at.own_col + i]);
        if (a.z) y[i] *= z[i] * sigmoid(z[i]);
        if (!inside) y[i] = 0.f;
      }
      store_some<W>(a.y + mine * a.ldy + own_safe, own_valid, y);
    }
  }
}

// One row of each sequence: row t is that of slot seq[t] (t without seq).
template <typename T, int LANES>
__global__ __launch_bounds__(256) void k_scan_step(Scan<T> a, int groups) {
  const int64_t t = blockIdx.x / groups;
  const int column = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  const int col = (int)(blockIdx.x % groups) * (256 / LANES) + column;
  const int slot = a.s.seq ? a.s.slot(t) : t < a.s.slots ? (int)t : -1;
  if (col >= a.n) return;
  float A[4], B[4], C[4], h[4] = {};
  load_A<T, LANES>(a, col, lane, A);
  const int k = min(lane * 4, a.states - 1);
  load_row_end<T, 4>(a.B + t * a.ldB + k, a.states - lane * 4, B);
  load_row_end<T, 4>(a.C + t * a.ldC + k, a.states - lane * 4, C);
  const int64_t at = ((int64_t)max(slot, 0) * a.n + col) * a.states;
  if (a.state && slot >= 0) load_row_end<float, 4>(a.state + at + k, a.states - lane * 4, h);
  const float u = (float)load_global<T>(a.u + t * a.ldu + col);
  const float x = (float)load_global<T>(a.dt + t * a.lddt + col) + (a.bias ? a.bias[col] : 0.f);
  float v;
  const float delta = softplus(x, v), du = delta * u;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h[i] = fmaf(__builtin_amdgcn_exp2f(delta * (A[i] * 1.44269504f)), h[i], du * B[i]);
    sum = fmaf(C[i], h[i], sum);
  }
  sum = column_sum<LANES>(sum);
  if (slot >= 0 && a.state_out)
    store_row<float, 4>(a.state_out + at + lane * 4, a.states - lane * 4, h);
  if (lane) return;
  float y = a.D ? fmaf(a.D[col], u, sum) : sum;
  if (a.z) {
    const float z = (float)load_global<T>(a.z + t * a.ldz + col);
    y *= z * sigmoid(z);
  }
  store_global<T>(a.y + t * a.ldy + col, (T)(slot >= 0 ? y : 0.f));
}

// ---------------------------------------------------------------------------------------------
// Backward
// ---------------------------------------------------------------------------------------------
template <int LANES>
struct ScanBackShared {
  static constexpr int kColumns = 256 / LANES;
  ScanShared<LANES> s;  // s.v: sum_n C h
  float p[kSpan][kColumns], gB[kSpan][kColumns], eA[kSpan][kColumns];
  float dBC[4][kSpan][2][4 * LANES];  // of the four waves
};

// dy silu(z), and dy silu'(z), of a row's own values.
template <typename T, int LANES>
__device__ __forceinline__ void scan_gate(const Scan<T>& a, int64_t t, int safe, int valid,
                                          float (&p)[ScanPlace<LANES>::kWide],
                                          float (&q)[ScanPlace<LANES>::kWide]) {
  constexpr int W = ScanPlace<LANES>::kWide;
  const int64_t row = min(t, a.s.rows - 1);
  load_some<W>(a.dy + row * a.lddy + safe, valid, p);
  if (!a.z) return;
  float z[W];
  load_some<W>(a.z + row * a.ldz + safe, valid, z);
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const float s = sigmoid(z[i]);
    q[i] = p[i] * s * fmaf(z[i], 1.f - s, 1.f);
    p[i] *= z[i] * s;
  }
}

// What a chunk adds to e^(delta A) g in front of it: links, local, deltas.
template <typename T, int LANES>
__global__ __launch_bounds__(256) void k_scan_back_local(Scan<T> a, int groups) {
  constexpr int W = ScanPlace<LANES>::kWide;
  __shared__ ScanShared<LANES> sh;  // v: p
  __shared__ int ends;
  const int chunk = blockIdx.x / groups + 1, group = blockIdx.x % groups;  // not the first chunk
  const ScanPlace<LANES> at(group);
  const int64_t first = (int64_t)chunk * a.chunk, end = min(first + a.chunk, a.s.rows);
  const int slot = a.s.slot(first);
  const bool goes_on = slot >= 0 && a.s.slot(first - 1) == slot;
  if (threadIdx.x == 0) ends = a.chunk;
  __syncthreads();
  if (goes_on)
    for (int i = threadIdx.x; i < end - first; i += 256)
      if (a.s.slot(first + i) != a.s.slot(first + i + 1)) atomicMin(&ends, i);
  __syncthreads();
  const bool whole = ends == a.chunk;
  if (group == 0 && threadIdx.x == 0)
    a.links[chunk] = goes_on ? kGoesOn | (whole ? kWhole : 0) : 0;
  if (!goes_on) return;
  const int64_t stop = whole ? end : first + ends + 1;  // behind the sequence's last row here
  const int column = threadIdx.x / LANES;
  const int own_at = at.first_col + at.own_col, own_safe = min(own_at, a.n - 1);
  const int own_valid = a.n - own_at;
  float A[4], g[4] = {}, bias[W] = {}, sum = 0.f;
  load_A<T, LANES>(a, at.col, at.lane, A);
#pragma unroll
  for (int i = 0; i < 4; ++i) A[i] *= 1.44269504f;
  if (a.bias) load_some<W>(a.bias + own_safe, own_valid, bias);
  for (int64_t t0 = (stop - 1) / kSpan * kSpan; t0 >= first; t0 -= kSpan) {
    const ScanOwn<W> own = scan_own<T, LANES>(a, at, t0);
    float p[W], q[W];
    scan_gate<T, LANES>(a, t0 + at.own_row, own_safe, own_valid, p, q);
    __syncthreads();
    scan_prepare<LANES>(at, own, bias, sh);
    scan_vectors<T, LANES>(a, t0, a.C, a.ldC, sh.C);
#pragma unroll
    for (int i = 0; i < W; ++i) sh.v[at.own_row][at.own_col + i] = p[i];
    __syncthreads();
    const int rows = (int)min((int64_t)kSpan, stop - t0);
    auto row = [&](int r) {
      const float delta = sh.delta[r][column], pr = sh.v[r][column];
      sum += delta;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        g[i] = __builtin_amdgcn_exp2f(delta * A[i]) * fmaf(sh.C[r][at.lane * 4 + i], pr, g[i]);
    };
    if (rows == kSpan) {
#pragma unroll
      for (int r = kSpan - 1; r >= 0; --r) row(r);
    } else {
      for (int r = rows - 1; r >= 0; --r) row(r);
    }
  }
  store_padded<LANES>(a.local, chunk, a.n, at.col, at.lane, g);
  if (at.lane == 0 && at.col < a.n) a.deltas[(int64_t)chunk * a.n + at.col] = sum;
}

// Sums of 8 values over the lanes of a wave that hold the same states of its columns: halves of the
// wave, then of the halves, exchange one of two values each.  Row k (of 16 lanes) ends up with
// values 2k and 2k + 1, in all its columns.
template <int LANES>
__device__ __forceinline__ void wave_sums(const float (&v)[8], float (&out)[2]) {
  float a[4], b[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[4 + i]),
                                                    false, false);
    a[i] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(a[i]), __float_as_uint(a[2 + i]),
                                                    false, false);
    b[i] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
  auto ror = [](float x, auto ctrl) {
    return __int_as_float(
        __builtin_amdgcn_update_dpp(0, __float_as_int(x), ctrl.value, 0xf, 0xf, true));
  };
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (LANES <= 8) b[i] += ror(b[i], std::integral_constant<int, 0x128>{});
    if constexpr (LANES <= 4) b[i] += ror(b[i], std::integral_constant<int, 0x124>{});
    if constexpr (LANES <= 2) b[i] += ror(b[i], std::integral_constant<int, 0x122>{});
    out[i] = b[i];
  }
}

template <typename T, int LANES>
__global__ __launch_bounds__(256) void k_scan_bwd(Scan<T> a, int groups) {
  constexpr int W = ScanPlace<LANES>::kWide, kOwn = kSpan / LANES, kStates = 4 * LANES;
  __shared__ ScanBackShared<LANES> sh;
  const int chunk = blockIdx.x / groups, group = blockIdx.x % groups;
  const ScanPlace<LANES> at(group);
  const int64_t first = (int64_t)chunk * a.chunk, end = min(first + a.chunk, a.s.rows);
  const int column = threadIdx.x / LANES, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int own_at = at.first_col + at.own_col, own_safe = min(own_at, a.n - 1);
  const int own_valid = a.n - own_at;
  float A[4], A2[4], g[4] = {}, dA[4] = {}, bias[W] = {}, D[W] = {}, dD[W] = {}, dbias[W] = {};
  load_A<T, LANES>(a, at.col, at.lane, A);
#pragma unroll
  for (int i = 0; i < 4; ++i) A2[i] = A[i] * 1.44269504f;
  if (a.bias) load_some<W>(a.bias + own_safe, own_valid, bias);
  if (a.D) load_some<W>(a.D + own_safe, own_valid, D);
  // g: e^(delta A) g of the row behind
  if (chunk + 1 < a.chunks && a.links[chunk + 1] & kGoesOn)
    load_padded<LANES>(a.local, chunk + 1, a.n, at.col, at.lane, g);
  for (int64_t t0 = (end - 1) / kSpan * kSpan; t0 >= first; t0 -= kSpan) {
    const int64_t mine = t0 + at.own_row;
    const ScanOwn<W> own = scan_own<T, LANES>(a, at, t0);
    float p[W], q[W];
    scan_gate<T, LANES>(a, mine, own_safe, own_valid, p, q);
    float h0[4];
    load_padded<LANES>(a.kept, t0 / kSpan, a.n, at.col, at.lane, h0);
    scan_prepare<LANES>(at, own, bias, sh.s);
    scan_vectors<T, LANES>(a, t0, a.B, a.ldB, sh.s.B);
    scan_vectors<T, LANES>(a, t0, a.C, a.ldC, sh.s.C);
    scan_rows<T, LANES>(a, t0, sh.s);
#pragma unroll
    for (int i = 0; i < W; ++i) sh.p[at.own_row][at.own_col + i] = p[i];
    __syncthreads();
    // the 16 rows' states again
    float h[kSpan][4], e[kSpan][4];  // h_t; e^(delta A)
    const bool plain = sh.s.plain;
#pragma unroll
    for (int r = 0; r < kSpan; ++r) {
      const float delta = sh.s.delta[r][column], du = sh.s.du[r][column];
      if (!plain && sh.s.flags[r] & kBegins) h0[0] = h0[1] = h0[2] = h0[3] = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        e[r][i] = __builtin_amdgcn_exp2f(delta * A2[i]);
        h0[i] = fmaf(e[r][i], h0[i], du * sh.s.B[r][at.lane * 4 + i]);
        h[r][i] = h0[i];
      }
    }
    load_padded<LANES>(a.kept, t0 / kSpan, a.n, at.col, at.lane, h0);
    float v[kOwn], gB[kOwn], eA[kOwn];
#pragma unroll
    for (int r = kSpan - 1; r >= 0; --r) {
      const int flags = plain ? kInside : sh.s.flags[r];
      float cs = 0.f, bs = 0.f, es = 0.f, out[8] = {};
      if (flags & kInside) {
        const float delta = sh.s.delta[r][column], du = sh.s.du[r][column];
        const float pr = sh.p[r][column];
        const bool begins = flags & kBegins;
        if (flags & kEnds) g[0] = g[1] = g[2] = g[3] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float C = sh.s.C[r][at.lane * 4 + i], B = sh.s.B[r][at.lane * 4 + i];
          g[i] = fmaf(C, pr, g[i]);
          cs = fmaf(C, h[r][i], cs);
          out[i] = g[i] * du;
          out[4 + i] = pr * h[r][i];
          bs = fmaf(g[i], B, bs);
          g[i] *= e[r][i];
          const float before = begins ? 0.f : r ? h[r ? r - 1 : 0][i] : h0[i];
          const float t = g[i] * before;
          es = fmaf(t, A[i], es);
          dA[i] = fmaf(t, delta, dA[i]);
        }
        if (at.col >= a.n)  // columns past the matrix have no part in the sums over columns
#pragma unroll
          for (int i = 0; i < 8; ++i) out[i] = 0.f;
      }
      cs = column_sum<LANES>(cs);
      bs = column_sum<LANES>(bs);
      es = column_sum<LANES>(es);
      const bool keep = at.lane == r % LANES;
      v[r / LANES] = keep || r % LANES == LANES - 1 ? cs : v[r / LANES];
      gB[r / LANES] = keep || r % LANES == LANES - 1 ? bs : gB[r / LANES];
      eA[r / LANES] = keep || r % LANES == LANES - 1 ? es : eA[r / LANES];
      float two[2];
      wave_sums<LANES>(out, two);
      if (lane % 16 < LANES) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int value = lane / 16 * 2 + i;
          sh.dBC[wave][r][value / 4][at.lane * 4 + value % 4] = two[i];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      sh.s.v[i * LANES + at.lane][column] = v[i];
      sh.gB[i * LANES + at.lane][column] = gB[i];
      sh.eA[i * LANES + at.lane][column] = eA[i];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kSpan * 2 * kStates; i += 256) {
      const int r = i / (2 * kStates), k = i % (2 * kStates);
      const float* w = &sh.dBC[0][r][0][0] + k;
      constexpr int kWave = kSpan * 2 * kStates;
      if (t0 + r < end)
        a.dBC[((int64_t)group * a.s.rows + t0 + r) * (2 * kStates) + k] =
            (w[0] + w[kWave]) + (w[2 * kWave] + w[3 * kWave]);
    }
    if (mine < end) {
      const bool inside = sh.s.flags[at.own_row] & kInside;
      float du[W], ddt[W], dz[W];
#pragma unroll
      for (int i = 0; i < W; ++i) {
        float w;
        const float x = own.dt[i] + bias[i], delta = softplus(x, w);
        const float sum_gB = sh.gB[at.own_row][at.own_col + i];
        du[i] = fmaf(delta, sum_gB, D[i] * p[i]);
        ddt[i] = fmaf(own.u[i], sum_gB, sh.eA[at.own_row][at.own_col + i]) * softplus_slope(x, w);
        dz[i] = q[i] * fmaf(D[i], own.u[i], sh.s.v[at.own_row][at.own_col + i]);
        if (!inside) du[i] = ddt[i] = dz[i] = 0.f;
        dD[i] += inside ? p[i] * own.u[i] : 0.f;
        dbias[i] += ddt[i];
      }
      store_some<W>(a.du + mine * a.lddu + own_safe, own_valid, du);
      store_some<W>(a.ddt + mine * a.ldddt + own_safe, own_valid, ddt);
      if (a.z) store_some<W>(a.dz + mine * a.lddz + own_safe, own_valid, dz);
    }
    __syncthreads();
  }
  store_padded<LANES>(a.dA, chunk, a.n, at.col, at.lane, dA);
  // dD and dbias over the 16 rows of a step, in order
#pragma unroll
  for (int i = 0; i < W; ++i) {
    sh.gB[at.own_row][at.own_col + i] = dD[i];
    sh.eA[at.own_row][at.own_col + i] = dbias[i];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < ScanPlace<LANES>::kColumns; i += 256) {
    if (at.first_col + i >= a.n) continue;
    float d = 0.f, b = 0.f;
#pragma unroll
    for (int r = 0; r < kSpan; ++r) {
      d += sh.gB[r][i];
      b += sh.eA[r][i];
    }
    a.dD[(int64_t)chunk * a.n + at.first_col + i] = d;
    a.dbias[(int64_t)chunk * a.n + at.first_col + i] = b;
  }
}

// dB and dC of a row: the sums of the groups' parts.
template <typename T>
__global__ __launch_bounds__(256) void k_scan_vectors(const float* __restrict__ part, int groups,
                                                      int64_t rows, int padded, int states,
                                                      T* __restrict__ dB, int64_t lddB,
                                                      T* __restrict__ dC, int64_t lddC) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = id / (2 * padded);
  const int k = (int)(id % (2 * padded));
  if (row >= rows) return;
  float sum = 0.f;
#pragma unroll 8
  for (int g = 0; g < groups; ++g)
    sum += load_global<float>(part + ((int64_t)g * rows + row) * (2 * padded) + k);
  if (k < states)
    store_global<T>(dB + row * lddB + k, (T)sum);
  else if (k >= padded && k - padded < states)
    store_global<T>(dC + row * lddC + k - padded, (T)sum);
}

// dA, dD and dbias: the sums of the chunks' parts, each NULL where it is not wanted.
__global__ __launch_bounds__(256) void k_scan_sums(const float* __restrict__ pA,
                                                   const float* __restrict__ pD,
                                                   const float* __restrict__ pb, int chunks, int n,
                                                   int padded, int states, float* __restrict__ dA,
                                                   float* __restrict__ dD,
                                                   float* __restrict__ dbias) {
  int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t all = (int64_t)n * padded;
  const float* p = pA;
  float* out = nullptr;
  int64_t ld = all;
  if (id < all) {
    const int k = (int)(id % padded);
    if (dA && k < states) out = dA + id / padded * states + k;
  } else if (id < all + n) {
    id -= all, ld = n, p = pD;
    if (dD) out = dD + id;
  } else if (id < all + 2 * (int64_t)n) {
    id -= all + n, ld = n, p = pb;
    if (dbias) out = dbias + id;
  }
  if (!out) return;
  float sum = 0.f;
#pragma unroll 8
  for (int c = 0; c < chunks; ++c) sum += load_global<float>(p + c * ld + id);
  *out = sum;
}

}  // namespace lm
