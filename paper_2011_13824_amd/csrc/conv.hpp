// Short causal convolution of every column, over sequences that lie behind each other.
//
//   pre_t = bias + sum_k w_k x_{t - taps + 1 + k},  y = act(pre)
//   dpre = dy act'(pre),  dx_t = sum_k w_k dpre_{t + taps - 1 - k}
//   dw_k = sum_t dpre_t x_{t - taps + 1 + k},  dbias = sum_t dpre_t
//
// In front of a sequence's first row stand the taps - 1 inputs of its state, or zeros.
//
// Bound by bytes.  A thread takes 16 bytes of columns (8 in the gradient) and walks over a strip of
// rows with the last taps - 1 inputs in registers, so that a row is read once, but for those in
// front of the strip, which its neighbour reads too and which come out of a cache.  The walk begins
// taps - 1 rows in front of the strip; a sequence that begins on the way replaces what the walk has
// met by its state.  The gradient walks on behind the strip's end, for the outputs that its last
// inputs reach, and adds a strip's part of dw and dbias in registers; the strips' parts are joined
// in order by k_sum_parts.
//
// 4 taps with silu: 8192 x 4096 bf16 33 us for 147 MB (4.4 TB/s, vector units 74 % busy), backward
// 55 + 8 us between events (201 MB read and written, and 26 MB of parts of dw and dbias twice; with
// 8 taps 105 + 15, of strips of 18 rows for 26); 4099 x 1001 f16 12 us forward, 22 + 5 backward, of
// which 64 rows take 4 and 9 + 2: the latency of a few loads in a row.  With 8 columns a thread the
// gradient's registers left two waves a SIMD (34 us for 24); with 8 rows ahead instead of 4 the
// forward pass took 52 us for 33.
#pragma once

#include "sequences.hpp"

namespace lm {

template <typename T>
struct Conv {
  const T *x, *w, *bias, *state, *dy;
  T *y, *state_out, *dx;
  float* part;  // [strips][taps + 1][n]: dw, dbias
  int64_t ldx, ldy, lddy, lddx;
  Sequences s;
  int n, strip, silu;
};

// The columns of a thread: 16 bytes forward; half of that in the gradient, whose sums take the
// registers.
template <typename T>
constexpr int kConvWide = 16 / sizeof(T);
template <typename T>
constexpr int kConvBackWide = kConvWide<T> / 2;

constexpr int kConvAhead = 4;  // rows on their way at a time

// W columns of rows as they are read: x[0 .. TAPS - 2] in front of the row, x[TAPS - 1] its own.
template <typename T, int TAPS, int W>
struct Window {
  Vec<T, W> x[TAPS];

  __device__ __forceinline__ void zero(int from, int to) {
#pragma unroll
    for (int k = 0; k < TAPS; ++k)
      if (k >= from && k < to)
#pragma unroll
        for (int i = 0; i < W; ++i) x[k][i] = (T)0.f;
  }
  // The inputs in front of a sequence's first row.
  __device__ __forceinline__ void front(const Conv<T>& a, int slot, const Columns<W>& c) {
    if (!a.state || slot < 0) return zero(0, TAPS - 1);
#pragma unroll
    for (int k = 0; k + 1 < TAPS; ++k)
      x[k] = load_columns<T, W>(a.state + ((int64_t)slot * (TAPS - 1) + k) * a.n, c);
  }
  __device__ __forceinline__ void shift() {
#pragma unroll
    for (int k = 0; k + 1 < TAPS; ++k) x[k] = x[k + 1];
  }
};

template <typename T, int TAPS, int W>
struct Taps {
  float w[TAPS][W], bias[W];

  __device__ __forceinline__ Taps(const Conv<T>& a, const Columns<W>& c) {
#pragma unroll
    for (int k = 0; k < TAPS; ++k)
      floats<T, W>(load_columns<T, W>(a.w + (int64_t)k * a.n, c), w[k]);
#pragma unroll
    for (int i = 0; i < W; ++i) bias[i] = 0.f;
    if (a.bias) floats<T, W>(load_columns<T, W>(a.bias, c), bias);
  }
  __device__ __forceinline__ void sum(const Window<T, TAPS, W>& in, float (&pre)[W]) const {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      pre[i] = bias[i];
#pragma unroll
      for (int k = 0; k < TAPS; ++k) pre[i] = fmaf(w[k][i], (float)in.x[k][i], pre[i]);
    }
  }
};

// A thread's strip and columns.
template <int W>
struct ConvPlace {
  int64_t strip, first, end;
  Columns<W> c;
  bool here;
  template <typename T>
  __device__ __forceinline__ explicit ConvPlace(const Conv<T>& a)
      : ConvPlace(a, piece_of<W>((int64_t)blockIdx.x * 256, (a.n + W - 1) / W)) {}
  template <typename T>
  __device__ __forceinline__ ConvPlace(const Conv<T>& a, Piece p)
      : strip(p.row),
        first(p.row * a.strip),
        end(min(p.row * a.strip + a.strip, a.s.rows)),
        c(p.col, a.n),
        here(p.row * a.strip < a.s.rows) {}
};

template <typename T, int TAPS>
__global__ __launch_bounds__(256) void k_conv_fwd(Conv<T> a) {
  constexpr int W = kConvWide<T>;
  const ConvPlace<W> at(a);
  if (!at.here) return;
  const Taps<T, TAPS, W> taps(a, at.c);
  Window<T, TAPS, W> in;
  in.zero(0, TAPS);
  int64_t t = max((int64_t)0, at.first - (TAPS - 1));
  int last = a.s.slot(t - 1);
  bool fresh = t == 0;  // the first row begins a sequence whatever stands before it
  for (; t < at.end; t += kConvAhead) {
    Vec<T, W> rows[kConvAhead];
    int slot[kConvAhead];
#pragma unroll
    for (int j = 0; j < kConvAhead; ++j) {
      const int64_t row = min(t + j, at.end - 1);
      slot[j] = a.s.slot(row);
      rows[j] = load_columns<T, W>(a.x + row * a.ldx, at.c);
    }
#pragma unroll
    for (int j = 0; j < kConvAhead; ++j) {
      if (t + j >= at.end) break;
      if (fresh || slot[j] != last) in.front(a, slot[j], at.c);
      fresh = false;
      last = slot[j];
      in.x[TAPS - 1] = rows[j];
      if (t + j >= at.first) {
        float y[W];
        taps.sum(in, y);
#pragma unroll
        for (int i = 0; i < W; ++i) {
          if (a.silu) y[i] *= sigmoid(y[i]);
          if (slot[j] < 0) y[i] = 0.f;
        }
        store_columns<T, W>(a.y + (t + j) * a.ldy, at.c, y);
      }
      in.shift();
    }
  }
}

// The last taps - 1 inputs of every sequence, its state's among them where it is shorter: block
// (pieces of 64 rows) x (columns).  It runs behind k_conv_fwd, so that state_out may be state: a
// thread reads what it replaces, and no other does.
template <typename T, int TAPS>
__global__ __launch_bounds__(256) void k_conv_state(Conv<T> a, int slabs) {
  constexpr int W = kConvWide<T>;
  const int64_t row0 = (int64_t)(blockIdx.x / slabs) * 64;
  const int col = ((int)(blockIdx.x % slabs) * 256 + threadIdx.x) * W;
  const int64_t mine = row0 + (threadIdx.x & 63);
  const int here = a.s.slot(mine);
  uint64_t ends = __ballot(here >= 0 && (mine + 1 == a.s.rows || a.s.slot(mine + 1) != here));
  if (col >= a.n) return;
  const Columns<W> c(col, a.n);
  for (; ends; ends &= ends - 1) {
    const int64_t t = row0 + __builtin_ctzll(ends);
    const int slot = a.s.slot(t);
    int64_t begin = t;  // of the sequence, as far back as its inputs are needed
    while (begin > 0 && begin > t - (TAPS - 1) && a.s.slot(begin - 1) == slot) --begin;
    Window<T, TAPS, W> now, old;
    old.front(a, slot, c);
#pragma unroll
    for (int k = 0; k + 1 < TAPS; ++k) {
      const int64_t from = t - (TAPS - 2) + k;
      if (from >= begin) {
        now.x[k] = load_columns<T, W>(a.x + from * a.ldx, c);
      } else {
        const int j = (int)(from - begin) + TAPS - 1;  // from the state's end
#pragma unroll
        for (int q = 0; q + 1 < TAPS; ++q)
          if (q == j) now.x[k] = old.x[q];
      }
    }
#pragma unroll
    for (int k = 0; k + 1 < TAPS; ++k) {
      float v[W];
      floats<T, W>(now.x[k], v);  // and back: exact
      store_columns<T, W>(a.state_out + ((int64_t)slot * (TAPS - 1) + k) * a.n, c, v);
    }
  }
}

// One row of each sequence: row t is that of slot seq[t] (t without seq).
template <typename T, int TAPS>
__global__ __launch_bounds__(256) void k_conv_step(Conv<T> a) {
  constexpr int W = kConvWide<T>;
  const Piece at = piece_of<W>((int64_t)blockIdx.x * 256, (a.n + W - 1) / W);
  if (at.row >= a.s.rows) return;
  const Columns<W> c(at.col, a.n);
  const int slot = a.s.seq ? a.s.slot(at.row) : at.row < a.s.slots ? (int)at.row : -1;
  Window<T, TAPS, W> in;
  in.x[TAPS - 1] = load_columns<T, W>(a.x + at.row * a.ldx, c);
  const Taps<T, TAPS, W> taps(a, c);
  in.front(a, slot, c);
  float y[W];
  taps.sum(in, y);
#pragma unroll
  for (int i = 0; i < W; ++i) {
    if (a.silu) y[i] *= sigmoid(y[i]);
    if (slot < 0) y[i] = 0.f;
  }
  store_columns<T, W>(a.y + at.row * a.ldy, c, y);
  if (!a.state_out || slot < 0) return;
#pragma unroll
  for (int k = 0; k + 1 < TAPS; ++k) {
    float v[W];
    floats<T, W>(in.x[k + 1], v);
    store_columns<T, W>(a.state_out + ((int64_t)slot * (TAPS - 1) + k) * a.n, c, v);
  }
}

// A strip's dx, and its part of dw and dbias.
template <typename T, int TAPS>
__global__ __launch_bounds__(256) void k_conv_bwd(Conv<T> a) {
  constexpr int W = kConvBackWide<T>;
  const ConvPlace<W> at(a);
  if (!at.here) return;
  const int64_t past = min(at.end + TAPS - 1, a.s.rows);  // rows whose outputs the strip reaches
  const Taps<T, TAPS, W> taps(a, at.c);
  Window<T, TAPS, W> in;
  in.zero(0, TAPS);
  // dx[j]: of row t - j, as far as it is known at row t
  float dx[TAPS][W] = {}, dw[TAPS][W] = {}, db[W] = {};
  int64_t t = max((int64_t)0, at.first - (TAPS - 1));
  int last = a.s.slot(t - 1), age = TAPS;  // rows since the sequence began, or more
  bool fresh = t == 0;
  auto put = [&](int64_t row, const float(&v)[W]) {
    if (row >= at.first && row < at.end) store_columns<T, W>(a.dx + row * a.lddx, at.c, v);
  };
  Vec<T, W> next_x[kConvAhead], next_dy[kConvAhead];
  int next_slot[kConvAhead];
  auto read = [&](int64_t from) {
#pragma unroll
    for (int j = 0; j < kConvAhead; ++j) {
      const int64_t row = min(from + j, past - 1);
      next_slot[j] = a.s.slot(row);
      next_x[j] = load_columns<T, W>(a.x + row * a.ldx, at.c);
      next_dy[j] = load_columns<T, W>(a.dy + row * a.lddy, at.c);
    }
  };
  read(t);
  for (; t < past; t += kConvAhead) {
    Vec<T, W> rows[kConvAhead], dy[kConvAhead];
    int slot[kConvAhead];
#pragma unroll
    for (int j = 0; j < kConvAhead; ++j)
      rows[j] = next_x[j], dy[j] = next_dy[j], slot[j] = next_slot[j];
    if (t + kConvAhead < past) read(t + kConvAhead);
#pragma unroll
    for (int j = 0; j < kConvAhead; ++j) {
      if (t + j >= past) break;
      ++age;
      if (fresh || slot[j] != last) {
        in.zero(0, TAPS - 1);
        age = 0;
      }
      fresh = false;
      last = slot[j];
      in.x[TAPS - 1] = rows[j];
#pragma unroll
      for (int k = TAPS - 1; k > 0; --k)
#pragma unroll
        for (int i = 0; i < W; ++i) dx[k][i] = dx[k - 1][i];
#pragma unroll
      for (int i = 0; i < W; ++i) dx[0][i] = 0.f;
      if (t + j >= at.first && slot[j] >= 0) {
        float pre[W], d[W];
        taps.sum(in, pre);
#pragma unroll
        for (int i = 0; i < W; ++i) {
          d[i] = (float)dy[j][i];
          if (a.silu) {
            const float p = sigmoid(pre[i]);
            d[i] *= p * fmaf(pre[i], 1.f - p, 1.f);
          }
        }
        auto reach = [&](int k) {
#pragma unroll
          for (int i = 0; i < W; ++i) dx[k][i] = fmaf(taps.w[TAPS - 1 - k][i], d[i], dx[k][i]);
        };
        if (age >= TAPS - 1) {
#pragma unroll
          for (int k = 0; k < TAPS; ++k) reach(k);
        } else {
#pragma unroll
          for (int k = 0; k < TAPS; ++k)
            if (k <= age) reach(k);
        }
        if (t + j < at.end) {
#pragma unroll
          for (int i = 0; i < W; ++i) db[i] += d[i];
#pragma unroll
          for (int k = 0; k < TAPS; ++k)
#pragma unroll
            for (int i = 0; i < W; ++i) dw[k][i] = fmaf(d[i], (float)in.x[k][i], dw[k][i]);
        }
      }
      put(t + j - (TAPS - 1), dx[TAPS - 1]);
      in.shift();
    }
  }
  // where the matrix ends with the strip, its last rows are still on their way
#pragma unroll
  for (int k = TAPS - 2; k >= 0; --k) put(past - 1 - k, dx[k]);
  float* part = a.part + at.strip * (TAPS + 1) * (int64_t)a.n;
#pragma unroll
  for (int k = 0; k < TAPS; ++k)
    store_columns<float, W>(part + (int64_t)k * a.n, at.c, dw[k]);
  store_columns<float, W>(part + (int64_t)TAPS * a.n, at.c, db);
}

}  // namespace lm
