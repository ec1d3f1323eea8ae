// Short causal convolution of every column, over sequences that lie behind each other.
//
//   pre_t = bias + sum_k w_k x_{t - taps + 1 + k},  y = act(pre)
//   dpre = dy act'(pre),  dx_t = sum_k w_k dpre_{t + taps - 1 - k}
//   dw_k = sum_t dpre_t x_{t - taps + 1 + k},  dbias = sum_t dpre_t
//
// In front of a sequence's first row stand the taps - 1 inputs of its state, or zeros.
//
// Bound by bytes.  A thread takes 8 columns and walks over a strip of rows with the last taps - 1
// inputs in registers, so that a row is read once, but for those in front of the strip, which its
// neighbour reads too and which come out of a cache.  The walk begins taps - 1 rows in front of the
// strip; a sequence that begins on the way replaces what the walk has met by its state.  The
// gradient walks on behind the strip's end, for the outputs that its last inputs reach, and adds a
// strip's part of dw and dbias in registers; the strips' parts are joined in order by k_sum_parts.
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

template <typename T>
__device__ __forceinline__ void load_taps(const Conv<T>& a, const T* p, int col, float (&v)[8]) {
  load_row_end<T, 8>(p + col, a.n - col, v);
}

// The inputs in front of a sequence's first row.
template <typename T, int TAPS>
__device__ __forceinline__ void front(const Conv<T>& a, int slot, int col, float (&x)[TAPS][8]) {
#pragma unroll
  for (int k = 0; k + 1 < TAPS; ++k)
    if (a.state && slot >= 0) {
      load_taps(a, a.state + ((int64_t)slot * (TAPS - 1) + k) * a.n, col, x[k]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[k][i] = 0.f;
    }
}

// x[0 .. TAPS - 2] are the inputs in front of the row, x[TAPS - 1] its own.
template <int TAPS>
__device__ __forceinline__ void conv_sum(const float (&x)[TAPS][8], const float (&w)[TAPS][8],
                                         const float (&bias)[8], float (&pre)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) pre[i] = bias[i];
#pragma unroll
  for (int k = 0; k < TAPS; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) pre[i] = fmaf(w[k][i], x[k][i], pre[i]);
}

template <typename T, int TAPS>
__device__ __forceinline__ void conv_weights(const Conv<T>& a, int col, float (&w)[TAPS][8],
                                             float (&bias)[8]) {
#pragma unroll
  for (int k = 0; k < TAPS; ++k) load_taps(a, a.w + (int64_t)k * a.n, col, w[k]);
#pragma unroll
  for (int i = 0; i < 8; ++i) bias[i] = 0.f;
  if (a.bias) load_taps(a, a.bias, col, bias);
}

template <int TAPS>
__device__ __forceinline__ void shift(float (&x)[TAPS][8]) {
#pragma unroll
  for (int k = 0; k + 1 < TAPS; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) x[k][i] = x[k + 1][i];
}

constexpr int kConvAhead = 4;  // rows on their way at a time

template <typename T, int TAPS>
__global__ __launch_bounds__(256) void k_conv_fwd(Conv<T> a) {
  const int per_row = (a.n + 7) / 8;
  const Piece at = piece_of((int64_t)blockIdx.x * 256, per_row);
  const int64_t first = at.row * a.strip, end = min(first + a.strip, a.s.rows);
  const int col = at.col;
  if (first >= a.s.rows) return;
  float w[TAPS][8], bias[8], x[TAPS][8] = {};
  conv_weights(a, col, w, bias);
  int64_t t = max((int64_t)0, first - (TAPS - 1));
  int last = a.s.slot(t - 1);
  bool fresh = t == 0;  // the first row begins a sequence whatever stands before it
  for (; t < end; t += kConvAhead) {
    float in[kConvAhead][8];
    int slot[kConvAhead];
#pragma unroll
    for (int j = 0; j < kConvAhead; ++j) {
      slot[j] = a.s.slot(min(t + j, end - 1));
      load_taps(a, a.x + min(t + j, end - 1) * a.ldx, col, in[j]);
    }
#pragma unroll
    for (int j = 0; j < kConvAhead; ++j) {
      if (t + j >= end) break;
      if (fresh || slot[j] != last) front<T, TAPS>(a, slot[j], col, x);
      fresh = false;
      last = slot[j];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[TAPS - 1][i] = in[j][i];
      if (t + j >= first) {
        float y[8];
        conv_sum<TAPS>(x, w, bias, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (a.silu) y[i] *= sigmoid(y[i]);
          if (slot[j] < 0) y[i] = 0.f;
        }
        store_row<T, 8>(a.y + (t + j) * a.ldy + col, a.n - col, y);
      }
      shift<TAPS>(x);
    }
  }
}

// The last taps - 1 inputs of every sequence, its state's among them where it is shorter: block
// (pieces of 64 rows) x (columns).  It runs behind k_conv_fwd, so that state_out may be state: a
// thread reads what it replaces, and no other does.
template <typename T, int TAPS>
__global__ __launch_bounds__(256) void k_conv_state(Conv<T> a, int slabs) {
  const int64_t row0 = (int64_t)(blockIdx.x / slabs) * 64;
  const int col = ((int)(blockIdx.x % slabs) * 256 + threadIdx.x) * 8;
  const int64_t mine = row0 + (threadIdx.x & 63);
  const int here = a.s.slot(mine);
  uint64_t ends = __ballot(here >= 0 && (mine + 1 == a.s.rows || a.s.slot(mine + 1) != here));
  if (col >= a.n) return;
  for (; ends; ends &= ends - 1) {
    const int64_t t = row0 + __builtin_ctzll(ends);
    const int slot = a.s.slot(t);
    int64_t begin = t;  // of the sequence, as far back as its inputs are needed
    while (begin > 0 && begin > t - (TAPS - 1) && a.s.slot(begin - 1) == slot) --begin;
    float x[TAPS][8], old[TAPS][8];
    front<T, TAPS>(a, slot, col, old);
#pragma unroll
    for (int k = 0; k + 1 < TAPS; ++k) {
      const int64_t from = t - (TAPS - 2) + k;
      if (from >= begin) {
        load_taps(a, a.x + from * a.ldx, col, x[k]);
      } else {
        const int j = (int)(from - begin) + TAPS - 1;  // from the state's end
#pragma unroll
        for (int q = 0; q + 1 < TAPS; ++q)
          if (q == j)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[k][i] = old[q][i];
      }
    }
#pragma unroll
    for (int k = 0; k + 1 < TAPS; ++k)
      store_row<T, 8>(a.state_out + ((int64_t)slot * (TAPS - 1) + k) * a.n + col, a.n - col, x[k]);
  }
}

// One row of each sequence: row t is that of slot seq[t] (t without seq).
template <typename T, int TAPS>
__global__ __launch_bounds__(256) void k_conv_step(Conv<T> a) {
  const Piece at = piece_of((int64_t)blockIdx.x * 256, (a.n + 7) / 8);
  if (at.row >= a.s.rows) return;
  const int col = at.col;
  const int slot = a.s.seq ? a.s.slot(at.row) : at.row < a.s.slots ? (int)at.row : -1;
  float w[TAPS][8], bias[8], x[TAPS][8], y[8];
  load_taps(a, a.x + at.row * a.ldx, col, x[TAPS - 1]);
  conv_weights(a, col, w, bias);
  front<T, TAPS>(a, slot, col, x);
  conv_sum<TAPS>(x, w, bias, y);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (a.silu) y[i] *= sigmoid(y[i]);
    if (slot < 0) y[i] = 0.f;
  }
  store_row<T, 8>(a.y + at.row * a.ldy + col, a.n - col, y);
  if (!a.state_out || slot < 0) return;
#pragma unroll
  for (int k = 0; k + 1 < TAPS; ++k)
    store_row<T, 8>(a.state_out + ((int64_t)slot * (TAPS - 1) + k) * a.n + col, a.n - col,
                    x[k + 1]);
}

// A strip's dx, and its part of dw and dbias.
template <typename T, int TAPS>
__global__ __launch_bounds__(256) void k_conv_bwd(Conv<T> a) {
  const int per_row = (a.n + 7) / 8;
  const Piece at = piece_of((int64_t)blockIdx.x * 256, per_row);
  const int64_t first = at.row * a.strip, end = min(first + a.strip, a.s.rows);
  const int64_t past = min(end + TAPS - 1, a.s.rows);  // rows whose outputs the strip reaches
  const int col = at.col;
  if (first >= a.s.rows) return;
  float w[TAPS][8], bias[8], x[TAPS][8] = {};
  // dx[j]: of row t - j, as far as it is known at row t
  float dx[TAPS][8] = {}, dw[TAPS][8] = {}, db[8] = {};
  conv_weights(a, col, w, bias);
  int64_t t = max((int64_t)0, first - (TAPS - 1));
  int last = a.s.slot(t - 1), age = t == 0 ? 0 : TAPS;  // rows since the sequence began, at least
  bool fresh = t == 0;
  auto put = [&](int64_t row, const float(&v)[8]) {
    if (row >= first && row < end) store_row<T, 8>(a.dx + row * a.lddx + col, a.n - col, v);
  };
  for (; t < past; t += kConvAhead) {
    float in[kConvAhead][8], dy[kConvAhead][8];
    int slot[kConvAhead];
#pragma unroll
    for (int j = 0; j < kConvAhead; ++j) {
      const int64_t row = min(t + j, past - 1);
      slot[j] = a.s.slot(row);
      load_taps(a, a.x + row * a.ldx, col, in[j]);
      load_taps(a, a.dy + row * a.lddy, col, dy[j]);
    }
#pragma unroll
    for (int j = 0; j < kConvAhead; ++j) {
      if (t + j >= past) break;
      ++age;
      if (fresh || slot[j] != last) {
#pragma unroll
        for (int k = 0; k + 1 < TAPS; ++k)
#pragma unroll
          for (int i = 0; i < 8; ++i) x[k][i] = 0.f;
        age = 0;
      }
      fresh = false;
      last = slot[j];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[TAPS - 1][i] = in[j][i];
#pragma unroll
      for (int k = TAPS - 1; k > 0; --k)
#pragma unroll
        for (int i = 0; i < 8; ++i) dx[k][i] = dx[k - 1][i];
#pragma unroll
      for (int i = 0; i < 8; ++i) dx[0][i] = 0.f;
      if (t + j >= first && slot[j] >= 0) {
        float pre[8], d[8];
        conv_sum<TAPS>(x, w, bias, pre);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          d[i] = dy[j][i];
          if (a.silu) {
            const float p = sigmoid(pre[i]);
            d[i] *= p * fmaf(pre[i], 1.f - p, 1.f);
          }
        }
        const bool own = t + j < end;
#pragma unroll
        for (int i = 0; i < 8; ++i) db[i] += own ? d[i] : 0.f;
#pragma unroll
        for (int k = 0; k < TAPS; ++k) {
          if (k > age) break;
#pragma unroll
          for (int i = 0; i < 8; ++i) dx[k][i] = fmaf(w[TAPS - 1 - k][i], d[i], dx[k][i]);
        }
        if (own)
#pragma unroll
          for (int k = 0; k < TAPS; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) dw[k][i] = fmaf(d[i], x[k][i], dw[k][i]);
      }
      put(t + j - (TAPS - 1), dx[TAPS - 1]);
      shift<TAPS>(x);
    }
  }
  // where the matrix ends with the strip, its last rows are still on their way
#pragma unroll
  for (int k = TAPS - 2; k >= 0; --k)
    put(past - 1 - k, dx[k]);
  if (!a.part) return;
  float* part = a.part + at.row * (TAPS + 1) * (int64_t)a.n + col;
#pragma unroll
  for (int k = 0; k < TAPS; ++k) store_row<float, 8>(part + (int64_t)k * a.n, a.n - col, dw[k]);
  store_row<float, 8>(part + (int64_t)TAPS * a.n, a.n - col, db);
}

}  // namespace lm
