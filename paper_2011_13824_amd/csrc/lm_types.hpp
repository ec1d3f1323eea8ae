// Element types, row accessors and 8-bit groups of the feed-forward block's kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace lm {

using bf16 = __bf16;
using f16 = _Float16;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// N elements of a row at any element alignment: one wide load or store (the hardware takes
// unaligned global accesses), where a typed vector access would promise an alignment that a
// tensor of odd width does not have.
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Vec {
  T v[N];
};

template <typename T, int N>
__device__ __forceinline__ void load_row(const T* p, int valid, float (&out)[N]) {
  if (valid >= N) {
    Vec<T, N> t = *reinterpret_cast<const Vec<T, N>*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = (float)t.v[i];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = i < valid ? (float)p[i] : 0.f;
  }
}

template <typename T, int N>
__device__ __forceinline__ void store_row(T* p, int valid, const float (&x)[N]) {
  if (valid >= N) {
    Vec<T, N> t;
#pragma unroll
    for (int i = 0; i < N; ++i) t.v[i] = (T)x[i];
    *reinterpret_cast<Vec<T, N>*>(p) = t;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < valid) p[i] = (T)x[i];
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

// x * 2^-e to the nearest whole number in [-127, 127]; any number for a NaN (the exponent marks
// its group).
__device__ __forceinline__ int to_int8(float x, float inverse) {
  return (int)__builtin_amdgcn_fmed3f(rintf(x * inverse), -127.f, 127.f);
}

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

}  // namespace lm
