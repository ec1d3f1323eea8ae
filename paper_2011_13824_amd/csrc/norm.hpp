// Root-mean-square norm with the residual's addition, forward and backward.
//
//   h = x + res,  rstd = (mean h^2 + eps)^-1/2,  y = w h rstd
//   dh = rstd (t - xhat mean(t xhat)) + dsum,  t = w dy,  xhat = h rstd;  dw = sum_rows dy xhat
//
// Bound by bytes, and by the launch where rows are few.  16384 x 4096 in bf16: forward with the
// 8-bit output 115 us for 0.6 GB (5.2 TB/s), backward 106 us for 0.54 GB (5.1 TB/s).  A row is read
// once, stays in registers (CH pieces of 8 columns a thread), is reduced over its THREADS threads
// and written.  Rows too wide for the registers of 1024 threads are read twice (CH = 0), the second
// time out of the caches.
#pragma once

#include "lm_types.hpp"

namespace lm {

// Sum over the THREADS threads that share a row; every thread gets it.  A row of one wave needs
// no barrier; otherwise `part` holds a sum per wave, and the barrier before the write keeps a
// wave of the next row from overwriting what a slower one still reads.
template <int THREADS>
__device__ __forceinline__ float row_sum(float v, float* part) {
#pragma unroll
  for (int s = 32; s; s >>= 1) v += __shfl_xor(v, s);
  if constexpr (THREADS > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) v += part[i];
  }
  return v;
}

template <typename T>
struct NormFwd {
  const T *x, *res, *w;
  int64_t ldx, ldr, lds, ldy;
  int64_t rows;
  int n;
  float eps;
  T *sum, *y;
  int8_t* q;
  uint8_t* exps;
  float* rstd;
};

// Writes one piece of h, y and the packed y.  `col` may lie past n (a thread without columns):
// the lanes of a group still meet in the exchange.
template <typename T>
__device__ __forceinline__ void norm_piece(const NormFwd<T>& a, int64_t row, int col,
                                           const float (&h)[8], float rstd, bool with_sum) {
  float y[8], w[8];
  load_row_end<T, 8>(a.w + col, a.n - col, w);
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = h[i] * rstd * w[i];
  if (with_sum && col < a.n) store_row<T, 8>(a.sum + row * a.lds + col, a.n - col, h);
  if (a.y && col < a.n) store_row<T, 8>(a.y + row * a.ldy + col, a.n - col, y);
  if (a.q) {
    const int e = group_exponent4(y);
    const int groups = groups_of(a.n);
    if (col < groups * kGroup) {
      store_global(a.q + row * groups * kGroup + col, pack8(y, e));
      if ((threadIdx.x & 3) == 0)
        store_global(a.exps + row * groups + col / kGroup, (uint8_t)e);
    }
  }
}

// THREADS threads a row (64: four rows a block), CH pieces of 8 columns each; CH = 0: any width.
template <typename T, int THREADS, int CH>
__global__ __launch_bounds__(THREADS == 64 ? 256 : THREADS) void k_norm_fwd(NormFwd<T> a) {
  __shared__ float part[THREADS / 64];
  constexpr int kRows = THREADS == 64 ? 4 : 1;
  const int t = THREADS == 64 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t row = (int64_t)blockIdx.x * kRows + (THREADS == 64 ? threadIdx.x >> 6 : 0);
  if (row >= a.rows) return;
  const T* x = a.x + row * a.ldx;
  const T* res = a.res ? a.res + row * a.ldr : nullptr;
  auto read = [&](int col, float(&h)[8]) {
    load_row_end<T, 8>(x + col, a.n - col, h);
    if (res) {
      float r[8];
      load_row_end<T, 8>(res + col, a.n - col, r);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] += r[i];
    }
  };
  float ss = 0.f;
  if constexpr (CH > 0) {
    float h[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) read((c * THREADS + t) * 8, h[c]);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) ss += h[c][i] * h[c][i];
    const float rstd = 1.f / sqrtf(row_sum<THREADS>(ss, part) / (float)a.n + a.eps);
    if (a.rstd && t == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int c = 0; c < CH; ++c)
      norm_piece(a, row, (c * THREADS + t) * 8, h[c], rstd, a.sum != nullptr);
  } else {
    const int span = (a.n + THREADS * 8 - 1) / (THREADS * 8) * (THREADS * 8);
    float h[8];
    for (int col = t * 8; col < span; col += THREADS * 8) {
      read(col, h);
#pragma unroll
      for (int i = 0; i < 8; ++i) ss += h[i] * h[i];
    }
    const float rstd = 1.f / sqrtf(row_sum<THREADS>(ss, part) / (float)a.n + a.eps);
    if (a.rstd && t == 0) a.rstd[row] = rstd;
    for (int col = t * 8; col < span; col += THREADS * 8) {
      read(col, h);
      norm_piece(a, row, col, h, rstd, a.sum != nullptr);
    }
  }
}

template <typename T>
struct NormBwd {
  const T *dy, *dsum, *h, *w;
  int64_t lddy, ldds, ldh, lddh;
  int64_t rows;
  int n;
  const float* rstd;
  T* dh;
  float* part;  // [blocks][n] sums of dy * xhat over a block's rows; NULL: no dw
};

// Columns col .. col + 7 of a row, 0 past its end, for k_norm_bwd.  CUT = false: n % 8 == 0, so a
// piece is whole or absent.  CUT = true: 32-bit elements one by one; of 16 bits the row's last eight
// where the end cuts a piece, moved down in registers, so that no branch keeps a row's loads from
// being on their way together (8192 bf16 rows of 4095 with dsum: 68 us, one by one 112; the 32-bit
// kernel's registers are all taken, and 2999 rows of 1001 took 13 us so, 11 one by one).
template <typename T, bool CUT>
__device__ __forceinline__ void load_piece(const T* row, int col, int n, float (&out)[8]) {
  const int valid = n - col;
  if constexpr (CUT && sizeof(T) == 2) {
    Vec<T, 8> t;
    if (n >= 8) {
      t = load_global<Vec<T, 8>>(row + min(col, n - 8));
      const int down = 8 - valid;  // of 1 .. 7; where it is 8 or more, nothing of t is kept
#pragma unroll
      for (int s = 4; s; s >>= 1)
#pragma unroll
        for (int i = 0; i + s < 8; ++i) t[i] = down > 0 && (down & s) ? t[i + s] : t[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] = load_global<T>(row + min(i, n - 1));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = i < valid ? (float)t[i] : 0.f;
  } else if constexpr (CUT) {
    load_row<T, 8>(row + col, valid, out);
  } else {
    const Vec<T, 8> t = load_global<Vec<T, 8>>(row + min(col, n - 8));
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = valid > 0 ? (float)t[i] : 0.f;
  }
}

// A block walks over rows (blockIdx.x, + gridDim.x, ...), keeps the sums of dy * xhat of its
// columns in registers and writes them once: dw needs no atomics, and its order is fixed by the
// sizes alone.  CH as above; CH = 0 takes rows of any width and leaves dw to k_norm_dw_wide.
template <typename T, int THREADS, int CH, bool CUT>
__global__ __launch_bounds__(THREADS == 64 ? 256 : THREADS) void k_norm_bwd(NormBwd<T> a) {
  __shared__ float part[THREADS / 64];
  constexpr int kRows = THREADS == 64 ? 4 : 1;
  constexpr int kCh = CH ? CH : 1;
  const int t = THREADS == 64 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t first = (int64_t)blockIdx.x * kRows + (THREADS == 64 ? threadIdx.x >> 6 : 0);
  const int64_t step = (int64_t)gridDim.x * kRows;
  const float inv_n = 1.f / (float)a.n;
  if constexpr (CH > 0) {
    float w[kCh][8], dw[kCh][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = (c * THREADS + t) * 8;
      load_piece<T, CUT>(a.w, col, a.n, w[c]);
#pragma unroll
      for (int i = 0; i < 8; ++i) dw[c][i] = 0.f;
    }
    for (int64_t row = first; row < a.rows; row += step) {
      const float rstd = a.rstd[row];
      float xhat[kCh][8], dy[kCh][8], dot = 0.f;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int col = (c * THREADS + t) * 8;
        load_piece<T, CUT>(a.h + row * a.ldh, col, a.n, xhat[c]);
        load_piece<T, CUT>(a.dy + row * a.lddy, col, a.n, dy[c]);
      }
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          xhat[c][i] *= rstd;
          dw[c][i] += dy[c][i] * xhat[c][i];
          dot += dy[c][i] * w[c][i] * xhat[c][i];
        }
      if (a.dh) {
        dot = row_sum<THREADS>(dot, part) * inv_n;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const int col = (c * THREADS + t) * 8;
          if (col >= a.n) continue;
          float d[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) d[i] = rstd * (dy[c][i] * w[c][i] - xhat[c][i] * dot);
          if (a.dsum) {
            float s[8];
            load_piece<T, CUT>(a.dsum + row * a.ldds, col, a.n, s);
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] += s[i];
          }
          store_row<T, 8>(a.dh + row * a.lddh + col, a.n - col, d);
        }
      }
    }
    if (!a.part) return;
    // the four waves of a block of one-wave rows hold sums of the same columns: added in order
    if constexpr (THREADS == 64) {
      __shared__ float all[4][64 * 8 * kCh];
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) all[threadIdx.x >> 6][(c * 64 + t) * 8 + i] = dw[c][i];
      __syncthreads();
      for (int col = threadIdx.x; col < a.n; col += 256)
        a.part[(int64_t)blockIdx.x * a.n + col] =
            (all[0][col] + all[1][col]) + (all[2][col] + all[3][col]);
    } else {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int col = (c * THREADS + t) * 8;
        if (col < a.n)
          store_row<float, 8>(a.part + (int64_t)blockIdx.x * a.n + col, a.n - col, dw[c]);
      }
    }
  } else {
    for (int64_t row = first; row < a.rows; row += step) {
      const float rstd = a.rstd[row];
      float h[8], dy[8], w[8], dot = 0.f;
      for (int col = t * 8; col < a.n; col += THREADS * 8) {
        load_row<T, 8>(a.h + row * a.ldh + col, a.n - col, h);
        load_row<T, 8>(a.dy + row * a.lddy + col, a.n - col, dy);
        load_row<T, 8>(a.w + col, a.n - col, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) dot += dy[i] * w[i] * (h[i] * rstd);
      }
      dot = row_sum<THREADS>(dot, part) * inv_n;
      for (int col = t * 8; col < a.n; col += THREADS * 8) {
        load_row<T, 8>(a.h + row * a.ldh + col, a.n - col, h);
        load_row<T, 8>(a.dy + row * a.lddy + col, a.n - col, dy);
        load_row<T, 8>(a.w + col, a.n - col, w);
        float s[8] = {};
        if (a.dsum) load_row<T, 8>(a.dsum + row * a.ldds + col, a.n - col, s);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] += rstd * (dy[i] * w[i] - h[i] * rstd * dot);
        store_row<T, 8>(a.dh + row * a.lddh + col, a.n - col, s);
      }
    }
  }
}

// Partial dw of rows wider than the registers hold: block (x, y) sums the rows y, y + gridDim.y,
// ... of 2048 columns.
template <typename T>
__global__ __launch_bounds__(256) void k_norm_dw_wide(NormBwd<T> a) {
  const int col = (blockIdx.x * 256 + threadIdx.x) * 8;
  if (col >= a.n) return;
  float dw[8] = {}, h[8], dy[8];
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const float rstd = a.rstd[row];
    load_row<T, 8>(a.h + row * a.ldh + col, a.n - col, h);
    load_row<T, 8>(a.dy + row * a.lddy + col, a.n - col, dy);
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[i] += dy[i] * (h[i] * rstd);
  }
  store_row<float, 8>(a.part + (int64_t)blockIdx.y * a.n + col, a.n - col, dw);
}

// dw = sum of the blocks' partial sums: a block takes 32 columns, each of its 32 groups of 8 threads
// every 32nd partial row, eight of them on their way at a time; the groups' sums are joined in
// order.  Bound by the latency of a few loads.
template <typename T>
__global__ __launch_bounds__(256) void k_norm_dw(const float* __restrict__ part, int blocks,
                                                 int n, T* __restrict__ dw) {
  __shared__ float all[32][33];
  const int c = threadIdx.x & 7, g = threadIdx.x >> 3, col = blockIdx.x * 32 + c * 4;
  float s[4] = {};
  int b = g;
  for (; b + 7 * 32 < blocks; b += 8 * 32) {
    float x[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      load_row<float, 4>(part + (int64_t)(b + i * 32) * n + col, n - col, x[i]);
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) s[k] += x[i][k];
  }
  for (; b < blocks; b += 32) {
    float x[4];
    load_row<float, 4>(part + (int64_t)b * n + col, n - col, x);
#pragma unroll
    for (int k = 0; k < 4; ++k) s[k] += x[k];
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) all[g][c * 4 + k] = s[k];
  __syncthreads();
  if (threadIdx.x >= 32 || blockIdx.x * 32 + threadIdx.x >= n) return;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) sum += all[i][threadIdx.x];
  dw[blockIdx.x * 32 + threadIdx.x] = (T)sum;
}

}  // namespace lm
