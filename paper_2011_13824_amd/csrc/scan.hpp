// Selective state space scan over sequences that lie behind each other, and its backward pass.
//
//   delta = softplus(dt + bias),  h_t = e^(delta A) h_{t-1} + delta u B_t   (a column, a state)
//   v_t = sum_n C_t h_t + D u,    y = v silu(z)
//
// and with p = dy silu(z), from the last row on:
//
//   g_t = C_t p_t + e^(delta_{t+1} A) g_{t+1},  e_t = g_t e^(delta_t A) h_{t-1}
//   dC_t = sum over columns of p h_t,  dB_t = sum over columns of g_t delta u
//   du = delta sum_n g B + D p,  ddelta = sum_n e A + u sum_n g B,  ddt = ddelta sigmoid(dt + bias)
//   dA = sum_t e delta,  dD = sum_t p u,  dbias = sum_t ddt,  dz = dy v silu'(z)
//
// Bound by the vector units: every row, column and state takes an exponential, which takes the time
// of two instructions, and four more instructions forward.  A column's states lie in LANES
// neighbouring lanes, four states each; a block takes 256 / LANES columns and walks over the rows by
// 16, of which it first computes what does not depend on the state (delta, delta u, and B and C as
// floats), one value a thread, into LDS.
//
// Rows are cut into chunks, so that there are enough blocks.  Before the real walk a first one
// computes what every chunk adds to a state that enters it with 0 (only for chunks whose last
// sequence goes on behind them, and from where that begins); the state that enters a chunk then
// follows from chunk to chunk, e^(A sum of delta) being what is left of the one before.  The
// gradient does the same from the last chunk on.  For it the forward pass keeps the state in front
// of every 16 rows, from which those 16 are computed again.
//
// 8192 rows of 4096 columns, 16 states, bf16: first walk 105 us (vector units full), link 9, real
// walk 182 (88 % busy; five instructions for a state, the exponential among them, 320 of a step's
// 560 are those); backward 115, 10 and 600 us (77 % busy, 1,870 instructions a step of 16 rows, two
// waves a SIMD), 12 for dB and dC, 5 for dA, dD and dbias.  These are a few calls behind an idle; in
// a run of 100 a forward pass takes 257 us, both 970.  64 states take 3.4 times as long as 16
// forward and 3.7 times in both passes.
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
  // per chunk: the state that a chunk adds, then the one that enters it; that of its last
  // sequence's begin; the sum of delta.  [chunks][n][4 * LANES], [chunks][n]; one flag a chunk
  float *local, *begin, *deltas;
  int *links;           // kGoesOn, kWhole
  float *dA, *dD, *dbias;  // [chunks][n][4 * LANES], [chunks][n]: parts
  float* dBC;           // [groups][rows][2][4 * LANES]: parts
};

// A chunk's last sequence goes on in the next (or, backwards, its first one comes from the chunk
// before); it fills the whole chunk, so that the state that enters is not replaced in it.
constexpr int kGoesOn = 1, kWhole = 2;

// log(1 + e^x) and, for its slope, v = e^-|x|.  The logarithm instruction is right to a unit in the
// last place, next to 1 too; what 1 + v loses of v is added again, where it counts (a small v), as
// it is.  Together at most 3.3 x 2^-24 of log(1 + v), for 2^22 values of v in each of eight octaves
// down to 2^-40.  (A series for the inverse hyperbolic tangent took 8 instructions more.)
__device__ __forceinline__ float softplus(float x, float& v) {
  v = __builtin_amdgcn_exp2f(fabsf(x) * -1.44269504f);
  const float w = 1.f + v;
  return fmaf(__builtin_amdgcn_logf(w), 0.693147181f, v - (w - 1.f)) + fmaxf(x, 0.f);
}
__device__ __forceinline__ float softplus_slope(float x, float v) {
  return (x >= 0.f ? 1.f : v) * __builtin_amdgcn_rcpf(1.f + v);
}

// The value as it is at this place: a last addition is else moved behind the branch that stores its
// sum, away from the lane exchange that it can be one instruction with.
__device__ __forceinline__ float here(float x) {
  asm volatile("" : "+v"(x));
  return x;
}

// The sum over the LANES neighbouring lanes of a column; each gets it.  The second half of the
// steps mirrors, which exchanges groups that already hold one value.
template <int LANES>
__device__ __forceinline__ float column_sum(float v) {
  auto dpp = [](float x, auto ctrl) {
    return __int_as_float(
        __builtin_amdgcn_mov_dpp(__float_as_int(x), ctrl.value, 0xf, 0xf, true));
  };
  v += dpp(v, std::integral_constant<int, 0xb1>{});  // quad_perm 1 0 3 2
  if constexpr (LANES > 2) v += dpp(v, std::integral_constant<int, 0x4e>{});   // 2 3 0 1
  if constexpr (LANES > 4) v += dpp(v, std::integral_constant<int, 0x141>{});  // row_half_mirror
  if constexpr (LANES > 8) v += dpp(v, std::integral_constant<int, 0x140>{});  // row_mirror
  return v;
}

// The columns and rows of a block and its threads.
template <int LANES>
struct ScanPlace {
  static constexpr int kColumns = 256 / LANES;
  static constexpr int kWide = kSpan / LANES;  // columns that a thread prepares of one row
  int col, lane;                               // of the walk
  int own_row, own_at;                         // of what the thread prepares: its first column,
  int own_slot;                                // and where that stands in LDS
  Columns<kWide> own;
  __device__ __forceinline__ ScanPlace(int group, int n)
      : col(group * kColumns + (int)threadIdx.x / LANES),
        lane(threadIdx.x % LANES),
        own_row((int)threadIdx.x / (kColumns / kWide)),
        own_at(group * kColumns + (int)threadIdx.x % (kColumns / kWide) * kWide),
        own_slot(kWide),
        own(own_at, n) {
    // a piece that is moved back may begin in front of the block's columns: kWide places are there
    own_slot += max(own.at - group * kColumns, -kWide);
  }
};

template <int LANES>
struct ScanShared {
  static constexpr int kColumns = 256 / LANES + kSpan / LANES, kStates = 4 * LANES;
  float2 step[kSpan][kColumns];  // delta, delta u; column j of the block stands at kWide + j
  __attribute__((aligned(16))) float B[kSpan][kStates];
  __attribute__((aligned(16))) float C[kSpan][kStates];
  int flags[kSpan], slot[kSpan], plain;  // plain: 16 rows inside one sequence
};

// What a thread reads for a step, ahead of it.
template <typename T, int LANES>
struct ScanNext {
  static constexpr int W = ScanPlace<LANES>::kWide;
  static constexpr int kEach = (kSpan * 4 * LANES + 255) / 256;
  Vec<T, W> u, dt, z, dy;
  T B[kEach], C[kEach];
  int slot[3];  // of the row, the one before and the one behind; by the first threads

  // WHAT: 1 u and dt, 2 z, 4 dy, 8 B, 16 C, 32 slots.  The step's first row is the block's, so that
  // a thread's place in it is a 32-bit offset.  Rows behind the last are the last, steps in front
  // of the first the first.
  template <int WHAT>
  __device__ __forceinline__ void read(const Scan<T>& a, const ScanPlace<LANES>& at, int64_t t) {
    const int64_t t0 = min(max(t, (int64_t)0), a.s.rows - 1);
    const int most = (int)min(a.s.rows - 1 - t0, (int64_t)(kSpan - 1));
    const int r = min(at.own_row, most);
    auto place = [](int row, int64_t ld) { return __umul24(row, (int)ld); };  // under 2^4, 2^22
    if constexpr (WHAT & 1) {
      u = load_columns<T, W>(a.u + t0 * a.ldu + place(r, a.ldu), at.own);
      dt = load_columns<T, W>(a.dt + t0 * a.lddt + place(r, a.lddt), at.own);
    }
    if constexpr (WHAT & 2)
      if (a.z) z = load_columns<T, W>(a.z + t0 * a.ldz + place(r, a.ldz), at.own);
    if constexpr (WHAT & 4) dy = load_columns<T, W>(a.dy + t0 * a.lddy + place(r, a.lddy), at.own);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int i = e * 256 + threadIdx.x;
      const int row = min(i / (4 * LANES), most), k = min(i % (4 * LANES), a.states - 1);
      if constexpr (WHAT & 8) B[e] = load_global<T>(a.B + t0 * a.ldB + place(row, a.ldB) + k);
      if constexpr (WHAT & 16) C[e] = load_global<T>(a.C + t0 * a.ldC + place(row, a.ldC) + k);
    }
    if constexpr (WHAT & 32)
      if (threadIdx.x < kSpan) {
        const int64_t row = t + threadIdx.x;
        slot[0] = a.s.slot(row);
        slot[1] = a.s.slot(row - 1);
        slot[2] = a.s.slot(row + 1);
      }
  }

  // B or C of 16 rows as floats, 0 behind the last state.
  __device__ __forceinline__ void put(const Scan<T>& a, const T (&v)[kEach],
                                      float (&out)[kSpan][4 * LANES]) const {
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int i = e * 256 + threadIdx.x, k = i % (4 * LANES);
      if (i < kSpan * 4 * LANES) out[i / (4 * LANES)][k] = k < a.states ? (float)v[e] : 0.f;
    }
  }

  __device__ __forceinline__ void put_rows(const Scan<T>& a, int64_t t0,
                                           ScanShared<LANES>& sh) const {
    if (threadIdx.x >= 64) return;
    int flags = 0;
    if (threadIdx.x < kSpan) {
      if (slot[0] >= 0) {
        flags = kInside;
        if (t0 + threadIdx.x == 0 || slot[1] != slot[0]) flags |= kBegins;
        if (slot[2] != slot[0]) flags |= kEnds;
      }
      sh.flags[threadIdx.x] = flags;
      sh.slot[threadIdx.x] = slot[0];
    }
    const uint64_t plain = __ballot(flags == kInside);
    if (threadIdx.x == 0) sh.plain = (plain & 0xffff) == 0xffff;
  }

  __device__ __forceinline__ void put_steps(const ScanPlace<LANES>& at, const float (&bias)[W],
                                            ScanShared<LANES>& sh) const {
    float sum[W];
    put_steps(at, bias, sh, false, sum);
  }
  // `counts`: the steps are added to sum.
  __device__ __forceinline__ void put_steps(const ScanPlace<LANES>& at, const float (&bias)[W],
                                            ScanShared<LANES>& sh, bool counts,
                                            float (&sum)[W]) const {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      float v;
      const float delta = softplus((float)dt[i] + bias[i], v);
      if (i < at.own.count)
        sh.step[at.own_row][at.own_slot + i] = make_float2(delta, delta * (float)u[i]);
      if (counts) sum[i] += delta;
    }
  }
};

// The sums of delta over a chunk, from those of the 16 rows of its steps, in order.
template <typename T, int LANES>
__device__ __forceinline__ void put_deltas(const Scan<T>& a, const ScanPlace<LANES>& at, int chunk,
                                           int group, const float (&sum)[ScanPlace<LANES>::kWide],
                                           ScanShared<LANES>& sh) {
  constexpr int W = ScanPlace<LANES>::kWide, kColumns = ScanPlace<LANES>::kColumns;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < W; ++i) sh.step[at.own_row][at.own_slot + i].x = sum[i];
  __syncthreads();
  const int col = group * kColumns + (int)threadIdx.x;
  if (threadIdx.x >= kColumns || col >= a.n) return;
  float d = 0.f;
#pragma unroll
  for (int r = 0; r < kSpan; ++r) d += sh.step[r][W + threadIdx.x].x;
  a.deltas[(int64_t)chunk * a.n + col] = d;
}

// Floats of the thread's own columns, 0 without p.
template <int LANES>
__device__ __forceinline__ void own_floats(const float* p, const ScanPlace<LANES>& at,
                                           float (&v)[ScanPlace<LANES>::kWide]) {
  constexpr int W = ScanPlace<LANES>::kWide;
#pragma unroll
  for (int i = 0; i < W; ++i) v[i] = 0.f;
  if (p) floats<float, W>(load_columns<float, W>(p, at.own), v);
}

// Four states of a column out of [n][states] (padded: [n][4 * LANES]), 0 behind the last.
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

// A, and A in powers of two.
template <typename T>
__device__ __forceinline__ void load_A(const Scan<T>& a, int col, int lane, float (&A)[4],
                                       float (&A2)[4]) {
  load_states(a.A, col, lane, a.states, a.n, A);
#pragma unroll
  for (int i = 0; i < 4; ++i) A2[i] = A[i] * 1.44269504f;
}

// A row's step of four states.
__device__ __forceinline__ void advance(float (&h)[4], float2 step, const float (&A2)[4],
                                        const float* B) {
  const f32x4 b = *(const f32x4*)B;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    h[i] = fmaf(__builtin_amdgcn_exp2f(step.x * A2[i]), h[i], step.y * b[i]);
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
  const ScanPlace<LANES> at(group, a.n);
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
  float A[4], A2[4], h[4] = {}, bias[W];
  load_A(a, at.col, at.lane, A, A2);
  own_floats<LANES>(a.bias, at, bias);
  if (from >= 0 && a.state) {
    load_states(a.state + (int64_t)slot * a.n * a.states, at.col, at.lane, a.states, a.n, h);
    store_padded<LANES>(a.begin, chunk, a.n, at.col, at.lane, h);
  }
  float sum[W] = {};
  const int64_t start = first + max(from, 0);
  int64_t t0 = start / kSpan * kSpan;
  const int column = W + (int)threadIdx.x / LANES;
  ScanNext<T, LANES> next;
  next.template read<1 | 8>(a, at, t0);
  for (; t0 < end; t0 += kSpan) {
    const int skip = (int)max((int64_t)0, start - t0);
    __syncthreads();
    next.put_steps(at, bias, sh, at.own_row >= skip, sum);
    next.put(a, next.B, sh.B);
    __syncthreads();
    next.template read<1 | 8>(a, at, t0 + kSpan);
    auto row = [&](int r) { advance(h, sh.step[r][column], A2, sh.B[r] + at.lane * 4); };
    if (skip == 0) {
#pragma unroll
      for (int r = 0; r < kSpan; ++r) row(r);
    } else {
      for (int r = skip; r < kSpan; ++r) row(r);
    }
  }
  store_padded<LANES>(a.local, chunk, a.n, at.col, at.lane, h);
  put_deltas(a, at, chunk, group, sum, sh);
}

// 2^x h, where 2^x by itself may be no float: over a chunk a state that is 0 stays 0 and a small one
// small, whatever an A over 0 makes of a state of 1.  Past 2^+-600 nothing is left to tell apart.
__device__ __forceinline__ float decayed(float h, float x) {
  x = __builtin_elementwise_minimum(__builtin_elementwise_maximum(x, -600.f), 600.f);
  const float whole = floorf(x);
  return __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f(x - whole) * h, (int)whole);
}

// The states that enter the chunks, in the place of what the chunks add: that of chunk c + 1 stands
// at c.  BACK: from the last chunk on; what enters chunk c from behind stands at c + 1.
template <typename T, int LANES, bool BACK>
__global__ __launch_bounds__(256) void k_scan_link(Scan<T> a) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int col = (int)(id / LANES), lane = (int)(id % LANES);
  if (col >= a.n) return;
  float A[4], A2[4], h[4] = {};
  load_A(a, col, lane, A, A2);
  constexpr int kAhead = 8;  // chunks whose values are on their way at a time
  for (int i0 = 0; i0 + 1 < a.chunks; i0 += kAhead) {
    float add[kAhead][4], sum[kAhead];
    int link[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int i = min(i0 + j, a.chunks - 2), c = BACK ? a.chunks - 1 - i : i;
      link[j] = load_global<int>(a.links + c);
      load_padded<LANES>(a.local, c, a.n, col, lane, add[j]);
      sum[j] = load_global<float>(a.deltas + (int64_t)c * a.n + col);
    }
    auto follow = [&](auto grows) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (i0 + j + 1 >= a.chunks) break;
        const int c = BACK ? a.chunks - 1 - (i0 + j) : i0 + j;
        const bool goes_on = link[j] & kGoesOn, whole = link[j] & kWhole;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          // what a chunk without a link holds was never written
          const float x = sum[j] * A2[k];
          const float left = !whole        ? 0.f
                             : grows.value ? decayed(h[k], x)
                                           : __builtin_amdgcn_exp2f(x) * h[k];
          h[k] = goes_on ? left + add[j][k] : 0.f;
        }
        if (goes_on) store_padded<LANES>(a.local, c, a.n, col, lane, h);
      }
    };
    // Without an A over 0 nothing grows.  8192 x 4096: 8.9 us; taking `decayed` for all 11.9, asking
    // before the first loads 11.1.
    if (A[0] > 0.f || A[1] > 0.f || A[2] > 0.f || A[3] > 0.f)
      follow(std::true_type{});
    else
      follow(std::false_type{});
  }
}

template <typename T, int LANES>
__global__ __launch_bounds__(256) void k_scan_fwd(Scan<T> a, int groups) {
  constexpr int W = ScanPlace<LANES>::kWide, kOwn = kSpan / LANES;
  __shared__ ScanShared<LANES> sh;
  __shared__ float shv[kSpan][ScanShared<LANES>::kColumns];  // sum_n C h
  const int chunk = blockIdx.x / groups;
  const ScanPlace<LANES> at(blockIdx.x % groups, a.n);
  const int64_t first = (int64_t)chunk * a.chunk, end = min(first + a.chunk, a.s.rows);
  const int column = W + (int)threadIdx.x / LANES;
  float A[4], A2[4], h[4] = {}, bias[W], D[W];
  load_A(a, at.col, at.lane, A, A2);
  own_floats<LANES>(a.bias, at, bias);
  own_floats<LANES>(a.D, at, D);
  if (chunk > 0 && a.links[chunk - 1] & kGoesOn)
    load_padded<LANES>(a.local, chunk - 1, a.n, at.col, at.lane, h);
  // the state of the sequence that goes on behind the chunk may have been replaced in the meantime,
  // where it goes to the place that it came from
  const bool goes_on = chunk + 1 < a.chunks && a.links[chunk] & kGoesOn;
  const int last_slot = goes_on ? a.s.slot(end - 1) : -1;
  ScanNext<T, LANES> next;
  next.template read<1 | 2 | 8 | 16 | 32>(a, at, first);
  for (int64_t t0 = first; t0 < end; t0 += kSpan) {
    const int64_t mine = t0 + at.own_row;
    next.put_steps(at, bias, sh);
    next.put(a, next.B, sh.B);
    next.put(a, next.C, sh.C);
    next.put_rows(a, t0, sh);
    const Vec<T, W> u = next.u, z = next.z;
    __syncthreads();
    next.template read<1 | 2 | 8 | 16 | 32>(a, at, t0 + kSpan);
    const bool inside = sh.flags[at.own_row] & kInside;
    if (a.kept) store_padded<LANES>(a.kept, t0 / kSpan, a.n, at.col, at.lane, h);
    float v[kOwn];
    auto row = [&](int r) {
      advance(h, sh.step[r][column], A2, sh.B[r] + at.lane * 4);
      const f32x4 c = *(const f32x4*)(sh.C[r] + at.lane * 4);
      float sum = c[0] * h[0];
#pragma unroll
      for (int i = 1; i < 4; ++i) sum = fmaf(c[i], h[i], sum);
      return column_sum<LANES>(sum);
    };
    if (sh.plain) {
#pragma unroll
      for (int r = 0; r < kSpan; ++r) {
        const float sum = row(r);
        v[r / LANES] = r % LANES == 0 || at.lane == r % LANES ? sum : v[r / LANES];
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
              load_states(a.state + (int64_t)slot * a.n * a.states, at.col, at.lane, a.states, a.n,
                          h);
          }
        }
        if (flags & kInside) sum = row(r);
        if (flags & kEnds && a.state_out && at.col < a.n)
          store_row<float, 4>(a.state_out + ((int64_t)slot * a.n + at.col) * a.states + at.lane * 4,
                              a.states - at.lane * 4, h);
        v[r / LANES] = r % LANES == 0 || at.lane == r % LANES ? sum : v[r / LANES];
      }
    }
#pragma unroll
    for (int i = 0; i < kOwn; ++i) shv[i * LANES + at.lane][column] = v[i];
    __syncthreads();
    if (mine < end && at.own_at < a.n) {
      float y[W];
#pragma unroll
      for (int i = 0; i < W; ++i) {
        y[i] = fmaf(D[i], (float)u[i], shv[at.own_row][at.own_slot + i]);
        if (a.z) y[i] *= (float)z[i] * sigmoid((float)z[i]);
        if (!inside) y[i] = 0.f;
      }
      store_columns<T, W>(a.y + mine * a.ldy, at.own, y);
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
  float A[4], A2[4], B[4], C[4], h[4] = {};
  load_A(a, col, lane, A, A2);
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
    h[i] = fmaf(__builtin_amdgcn_exp2f(delta * A2[i]), h[i], du * B[i]);
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

// p = dy silu(z) and q = dy silu'(z) of a row's own values.
template <typename T, int W>
__device__ __forceinline__ void scan_gate(bool gate, const Vec<T, W>& dy, const Vec<T, W>& z,
                                          float (&p)[W], float (&q)[W]) {
#pragma unroll
  for (int i = 0; i < W; ++i) {
    p[i] = (float)dy[i];
    if (gate) {
      const float x = (float)z[i], s = sigmoid(x);
      q[i] = p[i] * s * fmaf(x, 1.f - s, 1.f);
      p[i] *= x * s;
    }
  }
}

// What a chunk adds to e^(delta A) g in front of it: links, local, deltas.
template <typename T, int LANES>
__global__ __launch_bounds__(256) void k_scan_back_local(Scan<T> a, int groups) {
  constexpr int W = ScanPlace<LANES>::kWide;
  __shared__ ScanShared<LANES> sh;
  __shared__ float shp[kSpan][ScanShared<LANES>::kColumns];  // p
  __shared__ int ends;
  const int chunk = blockIdx.x / groups + 1, group = blockIdx.x % groups;  // not the first chunk
  const ScanPlace<LANES> at(group, a.n);
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
  const int column = W + (int)threadIdx.x / LANES;
  float A[4], A2[4], g[4] = {}, bias[W], sum[W] = {};
  load_A(a, at.col, at.lane, A, A2);
  own_floats<LANES>(a.bias, at, bias);
  int64_t t0 = (stop - 1) / kSpan * kSpan;
  ScanNext<T, LANES> next;
  next.template read<1 | 2 | 4 | 16>(a, at, t0);
  for (; t0 >= first; t0 -= kSpan) {
    float p[W], q[W];
    scan_gate<T, W>(a.z, next.dy, next.z, p, q);
    const int rows = (int)min((int64_t)kSpan, stop - t0);
    __syncthreads();
    next.put_steps(at, bias, sh, at.own_row < rows, sum);
    next.put(a, next.C, sh.C);
#pragma unroll
    for (int i = 0; i < W; ++i)
      if (i < at.own.count) shp[at.own_row][at.own_slot + i] = p[i];
    __syncthreads();
    next.template read<1 | 2 | 4 | 16>(a, at, t0 - kSpan);
    auto row = [&](int r) {
      const float delta = sh.step[r][column].x, pr = shp[r][column];
      const f32x4 c = *(const f32x4*)(sh.C[r] + at.lane * 4);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        g[i] = __builtin_amdgcn_exp2f(delta * A2[i]) * fmaf(c[i], pr, g[i]);
    };
    if (rows == kSpan) {
#pragma unroll
      for (int r = kSpan - 1; r >= 0; --r) row(r);
    } else {
      for (int r = rows - 1; r >= 0; --r) row(r);
    }
  }
  store_padded<LANES>(a.local, chunk, a.n, at.col, at.lane, g);
  put_deltas(a, at, chunk, group, sum, sh);
}

// Sums of 8 values over the lanes of a wave that hold the same states of its columns: halves of the
// wave, then of the halves, exchange one of two values each.  Row k (of 16 lanes) ends up with
// values 2k and 2k + 1, in all its columns.  (Products of the matrix units with ones, which add
// four lanes each, took the gradient of 8192 rows of 4096 columns from 0.60 to 0.79 ms.)
template <int LANES>
__device__ __forceinline__ void wave_sums(const float (&v)[8], float (&out)[2]) {
  float a[4], b[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]),
                                                    __float_as_uint(v[4 + i]), false, false);
    a[i] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(a[i]),
                                                    __float_as_uint(a[2 + i]), false, false);
    b[i] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
  auto ror = [](float x, auto ctrl) {
    return __int_as_float(
        __builtin_amdgcn_mov_dpp(__float_as_int(x), ctrl.value, 0xf, 0xf, true));
  };
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (LANES <= 8) b[i] += ror(b[i], std::integral_constant<int, 0x128>{});
    if constexpr (LANES <= 4) b[i] += ror(b[i], std::integral_constant<int, 0x124>{});
    if constexpr (LANES <= 2) b[i] += ror(b[i], std::integral_constant<int, 0x122>{});
    out[i] = here(b[i]);
  }
}

// The 16 rows of a step are taken in two halves, so that the states and decays of a half stay in
// registers between the walk to its end and the walk back; the state between the halves is computed
// first.
template <typename T, int LANES>
__global__ __launch_bounds__(256) void k_scan_bwd(Scan<T> a, int groups) {
  constexpr int W = ScanPlace<LANES>::kWide, kStates = 4 * LANES, kHalf = kSpan / 2;
  constexpr int kColumns = ScanShared<LANES>::kColumns;
  __shared__ ScanShared<LANES> sh;
  __shared__ float shp[kSpan][kColumns];       // p
  __shared__ f32x4 sums[kSpan][kColumns];      // over the states: C h, g B, e A
  __shared__ float dBC[4][kSpan][2][kStates];  // of the four waves
  const int chunk = blockIdx.x / groups, group = blockIdx.x % groups;
  const ScanPlace<LANES> at(group, a.n);
  const int64_t first = (int64_t)chunk * a.chunk, end = min(first + a.chunk, a.s.rows);
  const int column = W + (int)threadIdx.x / LANES, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float A[4], A2[4], g[4] = {}, dA[4] = {}, bias[W], D[W], dD[W] = {}, dbias[W] = {};
  load_A(a, at.col, at.lane, A, A2);
  own_floats<LANES>(a.bias, at, bias);
  own_floats<LANES>(a.D, at, D);
  // g: e^(delta A) g of the row behind
  if (chunk + 1 < a.chunks && a.links[chunk + 1] & kGoesOn)
    load_padded<LANES>(a.local, chunk + 1, a.n, at.col, at.lane, g);
  // Columns past the matrix have no part in the sums over columns: their delta u and p stay 0.
  for (int i = threadIdx.x; i < kSpan * kColumns; i += 256) {
    sh.step[i / kColumns][i % kColumns] = make_float2(0.f, 0.f);
    shp[i / kColumns][i % kColumns] = 0.f;
  }
  __syncthreads();
  int64_t t0 = (end - 1) / kSpan * kSpan;
  ScanNext<T, LANES> next;
  next.template read<1 | 2 | 4 | 8 | 16 | 32>(a, at, t0);
  float kept[4];
  load_padded<LANES>(a.kept, t0 / kSpan, a.n, at.col, at.lane, kept);
  for (; t0 >= first; t0 -= kSpan) {
    const int64_t mine = t0 + at.own_row;
    const Vec<T, W> u = next.u, dt = next.dt;
    float p[W], q[W], half_state[2][4];
    scan_gate<T, W>(a.z, next.dy, next.z, p, q);
    next.put_steps(at, bias, sh);
    next.put(a, next.B, sh.B);
    next.put(a, next.C, sh.C);
    next.put_rows(a, t0, sh);
#pragma unroll
    for (int i = 0; i < W; ++i)
      if (i < at.own.count) shp[at.own_row][at.own_slot + i] = p[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) half_state[0][i] = half_state[1][i] = kept[i];
    __syncthreads();
    next.template read<1 | 2 | 4 | 8 | 16 | 32>(a, at, t0 - kSpan);
    load_padded<LANES>(a.kept, max(t0 / kSpan - 1, (int64_t)0), a.n, at.col, at.lane, kept);
    auto walk = [&](auto plain) {
#pragma unroll
      for (int r = 0; r < kHalf; ++r) {
        if (!plain.value && sh.flags[r] & kBegins)
          half_state[1][0] = half_state[1][1] = half_state[1][2] = half_state[1][3] = 0.f;
        advance(half_state[1], sh.step[r][column], A2, sh.B[r] + at.lane * 4);
      }
#pragma unroll 1
      for (int half = 1; half >= 0; --half) {
        const int row0 = half * kHalf;
        float h[kHalf + 1][4], e[kHalf][4];  // the state in front of the half and behind its rows
#pragma unroll
        for (int i = 0; i < 4; ++i) h[0][i] = half ? half_state[1][i] : half_state[0][i];
#pragma unroll
        for (int r = 0; r < kHalf; ++r) {
          const float2 step = sh.step[row0 + r][column];
          const f32x4 b = *(const f32x4*)(sh.B[row0 + r] + at.lane * 4);
          // what is left of the state in front of a sequence's first row: nothing
          const bool begins = !plain.value && sh.flags[row0 + r] & kBegins;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            e[r][i] = begins ? 0.f : __builtin_amdgcn_exp2f(step.x * A2[i]);
            h[r + 1][i] = fmaf(e[r][i], begins ? 0.f : h[r][i], step.y * b[i]);
          }
        }
#pragma unroll
        for (int r = kHalf - 1; r >= 0; --r) {
          const int flags = plain.value ? kInside : sh.flags[row0 + r];
          float cs = 0.f, bs = 0.f, es = 0.f, out[8] = {};
          if (flags & kInside) {
            const float2 step = sh.step[row0 + r][column];
            const float pr = shp[row0 + r][column];
            const f32x4 b = *(const f32x4*)(sh.B[row0 + r] + at.lane * 4);
            const f32x4 c = *(const f32x4*)(sh.C[row0 + r] + at.lane * 4);
            const bool begins = flags & kBegins;
            if (flags & kEnds) g[0] = g[1] = g[2] = g[3] = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              g[i] = fmaf(c[i], pr, g[i]);
              cs = fmaf(c[i], h[r + 1][i], cs);
              out[i] = g[i] * step.y;
              out[4 + i] = pr * h[r + 1][i];
              bs = fmaf(g[i], b[i], bs);
              g[i] *= e[r][i];
              const float t = begins ? 0.f : g[i] * h[r][i];
              es = fmaf(t, A[i], es);
              dA[i] = fmaf(t, step.x, dA[i]);
            }
          }
          cs = here(column_sum<LANES>(cs));
          bs = here(column_sum<LANES>(bs));
          es = here(column_sum<LANES>(es));
          if (at.lane == 0) sums[row0 + r][column] = f32x4{cs, bs, es, 0.f};
          float two[2];
          wave_sums<LANES>(out, two);
          if (lane % 16 < LANES) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int value = lane / 16 * 2 + i;
              dBC[wave][row0 + r][value / 4][at.lane * 4 + value % 4] = two[i];
            }
          }
        }
      }
    };
    if (sh.plain)
      walk(std::true_type{});
    else
      walk(std::false_type{});
    __syncthreads();
    for (int i = threadIdx.x; i < kSpan * 2 * kStates; i += 256) {
      const int r = i / (2 * kStates), k = i % (2 * kStates);
      const int vec = k / kStates, state = k % kStates;
      if (t0 + r < end)
        a.dBC[((int64_t)group * a.s.rows + t0 + r) * (2 * kStates) + k] =
            (dBC[0][r][vec][state] + dBC[1][r][vec][state]) +
            (dBC[2][r][vec][state] + dBC[3][r][vec][state]);
    }
    if (mine < end && at.own_at < a.n) {
      const bool inside = sh.flags[at.own_row] & kInside;
      float du[W], ddt[W], dz[W];
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float x = (float)dt[i] + bias[i], ui = (float)u[i];
        const float v = __builtin_amdgcn_exp2f(fabsf(x) * -1.44269504f);
        const f32x4 s = sums[at.own_row][at.own_slot + i];
        du[i] = fmaf(sh.step[at.own_row][at.own_slot + i].x, s[1], D[i] * p[i]);
        ddt[i] = fmaf(ui, s[1], s[2]) * softplus_slope(x, v);
        dz[i] = q[i] * fmaf(D[i], ui, s[0]);
        if (!inside) du[i] = ddt[i] = dz[i] = 0.f;
        dD[i] += inside ? p[i] * ui : 0.f;
        dbias[i] += ddt[i];
      }
      store_columns<T, W>(a.du + mine * a.lddu, at.own, du);
      store_columns<T, W>(a.ddt + mine * a.ldddt, at.own, ddt);
      if (a.z) store_columns<T, W>(a.dz + mine * a.lddz, at.own, dz);
    }
    __syncthreads();
  }
  store_padded<LANES>(a.dA, chunk, a.n, at.col, at.lane, dA);
  // dD and dbias over the 16 rows of a step, in order
  if (at.own_at < a.n)
#pragma unroll
    for (int i = 0; i < W; ++i)
      sh.step[at.own_row][at.own_slot + i] = make_float2(dD[i], dbias[i]);
  __syncthreads();
  for (int i = threadIdx.x; i < ScanPlace<LANES>::kColumns; i += 256) {
    const int col = group * ScanPlace<LANES>::kColumns + i;
    if (col >= a.n) continue;
    float d = 0.f, b = 0.f;
#pragma unroll
    for (int r = 0; r < kSpan; ++r) {
      const float2 s = sh.step[r][W + i];
      d += s.x;
      b += s.y;
    }
    a.dD[(int64_t)chunk * a.n + col] = d;
    a.dbias[(int64_t)chunk * a.n + col] = b;
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
