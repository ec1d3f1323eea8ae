// Sequences that lie behind each other in the rows of a matrix, and sums of partial results.
//
// seq[t] is the sequence of row t, and the slot of its state; rows of a sequence are neighbours, so
// a sequence begins and ends where the number changes.  A number outside [0, slots) is padding.
// Without seq all rows are sequence 0.
#pragma once

#include "lm_types.hpp"

namespace lm {

struct Sequences {
  const int32_t* seq;
  int64_t rows;
  int slots;

  // The slot of row t, -1 for padding and outside the matrix.
  __device__ __forceinline__ int slot(int64_t t) const {
    if (t < 0 || t >= rows) return -1;
    if (!seq) return 0;
    const int s = load_global<int32_t>(seq + t);
    return s >= 0 && s < slots ? s : -1;
  }
};

// 1 / (1 + e^-x); e^-x may be infinite.
__device__ __forceinline__ float sigmoid(float x) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * -1.44269504f));
}

// out[i] = sum over b of part[b][i], b < blocks, rows ld apart; from column `split` on they are
// other's.  A block takes 32 columns, each of its 32 groups of 8 threads every 32nd row, eight of
// them on their way at a time; the groups' sums are joined in order.  Bound by the latency of a few
// loads.
template <typename T>
__global__ __launch_bounds__(256) void k_sum_parts(const float* __restrict__ part, int64_t blocks,
                                                   int64_t ld, int64_t n, int64_t split,
                                                   T* __restrict__ out, T* __restrict__ other) {
  __shared__ float all[32][33];
  const int c = threadIdx.x & 7, g = threadIdx.x >> 3;
  const int64_t col = (int64_t)blockIdx.x * 32 + c * 4;
  const int valid = (int)max((int64_t)0, min((int64_t)4, n - col));
  float s[4] = {};
  int64_t b = g;
  for (; b + 7 * 32 < blocks; b += 8 * 32) {
    float x[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i) load_row<float, 4>(part + (b + i * 32) * ld + col, valid, x[i]);
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) s[k] += x[i][k];
  }
  for (; b < blocks; b += 32) {
    float x[4];
    load_row<float, 4>(part + b * ld + col, valid, x);
#pragma unroll
    for (int k = 0; k < 4; ++k) s[k] += x[k];
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) all[g][c * 4 + k] = s[k];
  __syncthreads();
  const int64_t at = (int64_t)blockIdx.x * 32 + threadIdx.x;
  if (threadIdx.x >= 32 || at >= n) return;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) sum += all[i][threadIdx.x];
  (at < split ? out : other - split)[at] = (T)sum;
}

}  // namespace lm
