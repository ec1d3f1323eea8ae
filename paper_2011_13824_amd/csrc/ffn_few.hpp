// The feed-forward block for few tokens (a model that answers): every weight is read once.
//
//   h = act(x Wg^T) * (x Wu^T),  out = h Wd^T
//
// Bound by the weights' bytes, and by latency where they are small.  A block takes 16 features; its
// waves take the k axis in turn, 32 k a step, read the weights' rows straight into the registers of
// a 16-row matrix instruction (nothing is shared between waves, so LDS would add a trip), and add
// their sums in LDS in order.  Tokens fill the other side of the instruction, 16 at a time; lanes
// past the last one repeat it.  Weights are read where they lie at any alignment (by words and a
// shift off 4 bytes), and in 32 bits with the 32-bit instruction: three bf16 parts would be more
// bytes.  One token of 4096 x 10944 in bf16: 57 us, 4.7 TB/s of the 5.1 that a large copy reaches.
#pragma once

#include "ffn_tile.hpp"

namespace lm {

struct FewArgs {
  const void *A, *A2, *B;       // weights [I][K] (A2: Wu), tokens [J][K]
  int64_t lda, lda2, ldb, ldo;  // elements
  int I, J, K, gate;
  void* out;                    // [J][I]
};

// Eight k of a row and the products of one step.
template <typename T>
struct Eight {
  typename Mfma<T>::x8 v;
  __device__ __forceinline__ void load(const T* p) {
    v = load_global<Vec<T, 8>>(p);
  }
  __device__ __forceinline__ void load(const T* p, int valid) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < valid ? load_global<T>(p + i) : (T)0.f;
  }
  // From the words that hold the elements, each of which holds one at least.
  __device__ __forceinline__ void load_words(const T* p) {
    const int odd = (int)((uintptr_t)p >> 1) & 1;
    const T* words = p - odd;
    const Vec<uint32_t, 4> w = load_global<Vec<uint32_t, 4>>(words);
    const uint32_t last = load_global<uint32_t>(words + (odd ? 8 : 6));
    Vec<uint32_t, 4> r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      r[i] = __builtin_amdgcn_alignbit(i < 3 ? w[i < 3 ? i + 1 : 3] : last, w[i], 16 * odd);
    v = __builtin_bit_cast(typename Mfma<T>::x8, r);
  }
  static __device__ __forceinline__ f32x4 mac(const Eight& a, const Eight& b, f32x4 c) {
    return Mfma<T>::mac(a.v, b.v, c);
  }
};
template <>
struct Eight<float> {
  float v[8];
  __device__ __forceinline__ void load(const float* p) {
    const Vec<float, 8> t = load_global<Vec<float, 8>>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = t[i];
  }
  __device__ __forceinline__ void load(const float* p, int valid) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < valid ? load_global<float>(p + i) : 0.f;
  }
  static __device__ __forceinline__ f32x4 mac(const Eight& a, const Eight& b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[i], b.v[i], c, 0, 0, 0);
    return c;
  }
};

// TJ: groups of 16 tokens; UN: steps whose loads are in flight together; WORDS: rows of 16-bit
// weights that begin inside a 32-bit word are read by words and shifted.
template <typename T, bool GATE, int TJ, int WAVES, int UN, bool WORDS>
__global__ __launch_bounds__(WAVES * 64) void k_ffn_few(FewArgs a) {
  constexpr int kMats = GATE ? 2 : 1;
  __shared__ float part[WAVES][kMats][TJ][4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, q = lane >> 4;
  const int i0 = blockIdx.x * 16;
  const int64_t row = min(i0 + m, a.I - 1);
  const T* w[kMats];
  w[0] = (const T*)a.A + row * a.lda + q * 8;
  if constexpr (GATE) w[1] = (const T*)a.A2 + row * a.lda2 + q * 8;
  const T* x[TJ];
#pragma unroll
  for (int t = 0; t < TJ; ++t)
    x[t] = (const T*)a.B + (int64_t)min(t * 16 + m, a.J - 1) * a.ldb + q * 8;

  f32x4 acc[kMats][TJ];
#pragma unroll
  for (int c = 0; c < kMats; ++c)
#pragma unroll
    for (int t = 0; t < TJ; ++t) acc[c][t] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int full = a.K / 32;  // whole steps; wave w takes w, w + WAVES, ...
  for (int s = wave; s < full; s += UN * WAVES) {
    Eight<T> fw[UN][kMats], fx[UN][TJ];
#pragma unroll
    for (int n = 0; n < UN; ++n) {
      const int k = min(s + n * WAVES, full - 1) * 32;  // past the end: loaded, not multiplied
#pragma unroll
      for (int c = 0; c < kMats; ++c) {
        if constexpr (WORDS)
          fw[n][c].load_words(w[c] + k);
        else
          fw[n][c].load(w[c] + k);
      }
#pragma unroll
      for (int t = 0; t < TJ; ++t) {
        if constexpr (WORDS)
          fx[n][t].load_words(x[t] + k);
        else
          fx[n][t].load(x[t] + k);
      }
    }
#pragma unroll
    for (int n = 0; n < UN; ++n)
      if (s + n * WAVES < full) {
#pragma unroll
        for (int c = 0; c < kMats; ++c)
#pragma unroll
          for (int t = 0; t < TJ; ++t) acc[c][t] = Eight<T>::mac(fw[n][c], fx[n][t], acc[c][t]);
      }
  }
  if (full * 32 < a.K && wave == full % WAVES) {  // the last, partial step
    const int k = full * 32, valid = a.K - k - q * 8;
    Eight<T> fw[kMats], fx[TJ];
#pragma unroll
    for (int c = 0; c < kMats; ++c) fw[c].load(w[c] + k, valid);
#pragma unroll
    for (int t = 0; t < TJ; ++t) fx[t].load(x[t] + k, valid);
#pragma unroll
    for (int c = 0; c < kMats; ++c)
#pragma unroll
      for (int t = 0; t < TJ; ++t) acc[c][t] = Eight<T>::mac(fw[c], fx[t], acc[c][t]);
  }

#pragma unroll
  for (int c = 0; c < kMats; ++c)
#pragma unroll
    for (int t = 0; t < TJ; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) part[wave][c][t][r][lane] = acc[c][t][r];
  __syncthreads();
  // feature 4 (lane / 16) + r of token 16 t + lane % 16; 16 neighbouring threads write 16 features
  for (int o = threadIdx.x; o < TJ * 256; o += WAVES * 64) {
    const int t = o >> 8, j = (o >> 4) & 15, i = o & 15, from = (i >> 2) * 16 + j;
    float v[kMats];
#pragma unroll
    for (int c = 0; c < kMats; ++c) {
      v[c] = 0.f;
#pragma unroll
      for (int p = 0; p < WAVES; ++p) v[c] += part[p][c][t][i & 3][from];
    }
    if constexpr (GATE) {
      float act, slope;
      gate_fn(a.gate, sizeof(T) == 2, v[0], act, slope);
      v[0] = act * v[1];
    }
    const int64_t token = t * 16 + j;
    if (token < a.J && i0 + i < a.I) ((T*)a.out)[token * a.ldo + i0 + i] = (T)v[0];
  }
}

}  // namespace lm
