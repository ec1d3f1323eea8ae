// Element types, row accessors and 8-bit groups of the feed-forward block's kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace lm {

using bf16 = __bf16;
using f16 = _Float16;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// N elements of a row at any element alignment: one wide load or store (the hardware takes
// unaligned global accesses), where a plain vector type would promise an alignment that a tensor
// of odd width does not have.
template <typename T, int N>
using Vec = T __attribute__((ext_vector_type(N), aligned(sizeof(T))));

// Global memory: a pointer that comes out of an array in a kernel's arguments is otherwise taken
// for one that may point anywhere, and its accesses for LDS traffic too.
template <typename V>
__device__ __forceinline__ V load_global(const void* p) {
  return *(const __attribute__((address_space(1))) V*)p;
}
template <typename V>
__device__ __forceinline__ void store_global(void* p, V v) {
  *(__attribute__((address_space(1))) V*)p = v;
}

template <typename T, int N>
__device__ __forceinline__ void load_row(const T* p, int valid, float (&out)[N]) {
  if (valid >= N) {
    const Vec<T, N> t = load_global<Vec<T, N>>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = (float)t[i];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = i < valid ? (float)load_global<T>(p + i) : 0.f;
  }
}

// The same where few registers are live: past the row's end its last element is read again, so that
// no branch stands between the loads and the lane waits for them once.  Against load_row, bf16
// and 8192 rows: the norm's forward pass of 4095 columns 60 for 77 us, packing 5165 28 for 31 us.
// The norm's gradient, whose registers are all taken, went from 57 to 87 us and reads otherwise.
template <typename T, int N>
__device__ __forceinline__ void load_row_end(const T* p, int valid, float (&out)[N]) {
  if (valid >= N || valid <= 0) return load_row<T, N>(p, valid, out);
  T t[N];
#pragma unroll
  for (int i = 0; i < N; ++i) t[i] = load_global<T>(p + min(i, valid - 1));
#pragma unroll
  for (int i = 0; i < N; ++i) out[i] = i < valid ? (float)t[i] : 0.f;
}

template <typename T, int N>
__device__ __forceinline__ void store_row(T* p, int valid, const float (&x)[N]) {
  Vec<T, N> t;
#pragma unroll
  for (int i = 0; i < N; ++i) t[i] = (T)x[i];
  if (valid >= N) {
    store_global(p, t);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < valid) store_global<T>(p + i, t[i]);
  }
}

// ---------------------------------------------------------------------------------------------
// 8 bits: int8 [rows][groups * 32], then a biased exponent [rows][groups]
// ---------------------------------------------------------------------------------------------
constexpr int kGroup = 32;
constexpr int kLeastExp = -120;  // the scale and its reciprocal are both normal floats
constexpr int kMostExp = 121;     // 127 * 2^e is finite; what lies beyond is held as that
constexpr int kNoValue = 255;    // the exponent byte of a group that holds an infinity or a NaN

__host__ __device__ __forceinline__ int groups_of(int n) { return (n + kGroup - 1) / kGroup; }

// Biased exponent of a group's scale from the bits of its largest magnitude m * 2^k, 1 <= m < 2:
// e = k - 6 where m <= 127/64, k - 5 above; an infinity's or a NaN's bits compare above every
// finite value's, so the maximum of the bits finds them too.
__device__ __forceinline__ int group_exponent(uint32_t top) {
  if (top >= 0x7f800000u) return kNoValue;
  int k = (int)(top >> 23) - 127;
  int e = k - 6 + ((top & 0x7fffffu) > 0x7e0000u);
  return min(max(e, kLeastExp), kMostExp) + 127;
}

// 2^-e and 2^e of a biased exponent; a group without values reads back as NaN.
__device__ __forceinline__ float group_inverse(int biased) {
  return biased == kNoValue ? 0.f : __uint_as_float((uint32_t)(254 - biased) << 23);
}
__device__ __forceinline__ float group_scale(int biased) {
  return biased == kNoValue ? __uint_as_float(0x7fc00000u)
                            : __uint_as_float((uint32_t)biased << 23);
}

// The largest magnitude of eight values; a NaN among them is the result.
__device__ __forceinline__ float largest8(const float (&x)[8]) {
  float m = fabsf(x[0]);
#pragma unroll
  for (int i = 1; i < 8; ++i) m = __builtin_elementwise_maximum(m, fabsf(x[i]));
  return m;
}

// Biased exponent of the group that four neighbouring lanes hold, eight values each.
__device__ __forceinline__ int group_exponent4(const float (&x)[8]) {
  // the sign is off, so the bits order as the values do, and a NaN comes last
  uint32_t top = __float_as_uint(largest8(x)) & 0x7fffffffu;
  top = max(top, (uint32_t)__shfl_xor((int)top, 1));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2));
  return group_exponent(top);
}

// Eight values as multiples of 2^e, rounded to the nearest (ties to even) by the addition of
// 1.5 * 2^23: the sum's low byte is the multiple in two's complement.  Only under the largest
// exponent a multiple can pass 127.  In a group without values any byte comes out.
__device__ __forceinline__ u32x2 pack8(const float (&x)[8], int biased) {
  constexpr float kWhole = 12582912.f;
  const float inv = group_inverse(biased);
  uint32_t b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(fmaf(x[i], inv, kWhole));
  if (biased == kMostExp + 127) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      b[i] = (uint32_t)(int)__builtin_amdgcn_fmed3f(rintf(x[i] * inv), -127.f, 127.f);
  }
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    // bytes 0 of two words side by side, then of both pairs
    const uint32_t lo = __builtin_amdgcn_perm(b[4 * h + 1], b[4 * h], 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(b[4 * h + 3], b[4 * h + 2], 0x0c0c0400u);
    w[h] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
  }
  return u32x2{w[0], w[1]};
}

// Eight multiples as values.
__device__ __forceinline__ void unpack8(u32x2 w, int biased, float (&x)[8]) {
  const float s = group_scale(biased);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)(int8_t)(w[i >> 2] >> 8 * (i & 3)) * s;
}

// The same for values that are stored as T.  A finite value can pass f16's range: magnitudes from
// 65024 on are held as 64 * 2^10.  They become its largest, which is the nearer one to what was
// packed; a NaN stays one.
template <typename T>
__device__ __forceinline__ void unpack8_as(u32x2 w, int biased, float (&x)[8]) {
  unpack8(w, biased, x);
  if constexpr (__is_same(T, f16)) {
    constexpr float kMost = 65504.f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (fabsf(x[i]) > kMost) x[i] = copysignf(kMost, x[i]);
  }
}

}  // namespace lm
